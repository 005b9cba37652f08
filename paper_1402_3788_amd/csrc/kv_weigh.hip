// The weight that attention gave to cached positions.
//
// A wave takes a tile of 32 positions of a sequence, looks their keys up once from the
// centres of its head in LDS, which become the rows of one operand of
// v_mfma_f32_32x32x16, and goes through the rows of the sequence's new tokens (the query
// heads of each), 32 at a time as columns of the other: exp(z - lse) is summed for each
// position in its lanes, and over the lanes at the end. Each sum has one order and one
// writer. The keys' codes are the bytes that must come from memory; for a single new token
// they bound it, for many the exponentials do.
#include "kv_tokens_device.h"

namespace lloyd {

namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;


template <int D, int SUB>
struct Form {
    static constexpr int S = D / SUB, H = S / 2;         // codes of a key, of a lane's half of it
    static constexpr int kBook = D * 512;                // [S][256][SUB]
};

// N bytes of codes, in whole words.
template <int N>
__device__ inline void load_codes(uint32_t (&dst)[(N + 3) / 4], const uint8_t *src)
{
    constexpr int align = N % 16 == 0 ? 16 : N % 8 == 0 ? 8 : N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1;
    dst[(N - 1) / 4] = 0;
    __builtin_memcpy(dst, __builtin_assume_aligned(src, align), N);
}

template <int D, int SUB, bool FP16>
__global__ __launch_bounds__(kThreads, 4) void kv_weigh_kernel(KvCache c, KvNew a, KvWeigh w, int splits)
{
    using F = Form<D, SUB>;
    extern __shared__ uint4 lds[];
    char *const book = reinterpret_cast<char *>(lds);
    int *const first = reinterpret_cast<int *>(book + F::kBook);         // [seqs + 1]
    __shared__ int wave_sum[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int h = blockIdx.x % c.heads, j = blockIdx.x / c.heads;
    const int heads = c.heads * a.group;
    const int64_t wrow = (int64_t)h * w.weights_head;

    // The centres of this head's keys, entries from K up zeros.
    const uint16_t *const from = c.k_centres + (int64_t)h * F::S * c.K * SUB;
    if (c.K == 256) {
#pragma unroll
        for (int i = 0; i < D * 32 / kThreads; ++i)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)(reinterpret_cast<const char *>(from) + (i * kThreads + tid) * 16),
                (__attribute__((address_space(3))) void *)(book + (i * kThreads + (wave << 6)) * 16), 16, 0, 0);
    } else {
        for (int i = tid; i < F::S * 256; i += kThreads) {
            KvEntry<SUB> e{};
            if ((i & 255) < c.K) e = kv_load<SUB>(from + ((i >> 8) * c.K + (i & 255)) * SUB);
            reinterpret_cast<KvEntry<SUB> *>(book)[i] = e;
        }
    }
    // A sequence's tiles, and where each one's begin among all. One without new tokens has
    // none, and a window leaves out those before it.
    const int span = (int)min(w.positions, (int64_t)a.table_pages << c.page_log2);
    const auto tile0_of = [&](const KvSeq &s) {
        return a.window ? max(s.len - s.n - a.window + 1, 0) >> 5 : 0;
    };
    const auto tiles_of = [&](int b) {
        const KvSeq s = kv_seq(c, a, b);
        return s.n ? max(((min(s.len, span) + 31) >> 5) - tile0_of(s), 0) : 0;
    };
    int tiles;
    {
        const int per = (a.seqs + kThreads - 1) / kThreads;
        int sum = 0;
        for (int k = 0; k < per; ++k)
            if (tid * per + k < a.seqs) sum += tiles_of(tid * per + k);
        const int upto = scan_lanes(sum);
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        int at = upto - sum;
        tiles = 0;
        for (int i = 0; i < kWaves; ++i) {
            if (i < wave) at += wave_sum[i];
            tiles += wave_sum[i];
        }
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            if (b >= a.seqs) break;
            first[b] = at;
            at += tiles_of(b);
        }
        if (tid == 0) first[a.seqs] = tiles;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the centres
    __syncthreads();
    // What no tile covers.
    if (!w.add) {
        for (int b = j; b < a.seqs; b += splits) {
            float *const to = w.weights + b * w.weights_seq + wrow;
            const int n = first[b + 1] - first[b], tile0 = n ? tile0_of(kv_seq(c, a, b)) : 0;
            for (int i = tid; i < tile0 * 32; i += kThreads) to[i] = 0.f;
            for (int64_t i = (int64_t)(tile0 + n) * 32 + tid; i < w.positions; i += kThreads) to[i] = 0.f;
        }
    }

    const unsigned page_bytes = (unsigned)(c.heads * F::S) << c.page_log2;
    const unsigned last_page = (unsigned)min(c.pages - 1, (int64_t)0x7FFFFFFF);
    const unsigned pm = (1u << c.page_log2) - 1;
    const uint8_t *const lane_codes = c.k_codes + (((int64_t)h * F::S) << c.page_log2) + half * F::H;
    const bool changed = a.cap_log2 > 0.f || a.slopes;
    const int step = kWaves * splits;

    // Tile t: its sequence, and a lane's position and page.
    struct Where {
        int b, pos, page;
    };
    const auto find = [&](int t, int b) {
        Where x;
        // the last sequence whose tiles begin at t or before: of 64 after b at a time
        for (;;) {
            const int n = b + 1 + lane;
            const int more = __popcll(__ballot(n < a.seqs && first[min(n, a.seqs)] <= t));
            b += more;
            if (more < kWave) break;
        }
        x.b = __builtin_amdgcn_readfirstlane(b);
        const KvSeq s = kv_seq(c, a, x.b);
        x.pos = (t - __builtin_amdgcn_readfirstlane(first[x.b]) + tile0_of(s)) * 32;
        x.page = a.table[x.b * a.table_stride + (min(x.pos + col, s.len - 1) >> c.page_log2)];
        return x;
    };
    const auto load = [&](uint32_t (&codes)[(F::H + 3) / 4], const Where &x) {
        load_codes<F::H>(codes, lane_codes + (uint64_t)min((unsigned)x.page, last_page) * page_bytes +
                                    (((unsigned)x.pos + col) & pm) * F::S);
    };
    int t = j * kWaves + wave;
    if (t >= tiles) return;
    Where now = find(t, 0), next = now;
    uint32_t codes[(F::H + 3) / 4];
    load(codes, now);
    if (t + step < tiles) next = find(t + step, now.b);
    for (; t < tiles; t += step) {
        // the keys: a lane has features [half D / 2, + D / 2) of position col
        u4v k[D / 16];
        {
            KvEntry<SUB> e[F::H];
            const char *const at = book + half * (F::H * 512 * SUB);
#pragma unroll
            for (int n = 0; n < F::H; ++n)
                e[n] = *reinterpret_cast<const KvEntry<SUB> *>(
                    at + n * (512 * SUB) + (codes[n / 4] >> (8 * (n % 4)) & 255) * (2 * SUB));
            __builtin_memcpy(k, e, sizeof(k));
        }
        const Where x = now;
        now = next;
        if (t + step < tiles) load(codes, now);
        if (t + 2 * step < tiles) next = find(t + 2 * step, now.b);

        const KvSeq s = kv_seq(c, a, x.b);
        const int rows = s.n * a.group;
        float sum[16] = {};
        for (int r0 = 0; r0 < rows; r0 += 32) {
            const int row = r0 + col;
            const int tok = (int)((unsigned)row / (unsigned)a.group), hq = h * a.group + (int)((unsigned)row % (unsigned)a.group);
            KvSeen seen{0, 0, 0};
            float lse = INFINITY;
            if (row < rows) {
                seen = kv_seen(a, s, tok);
                lse = w.lse[(int64_t)(s.t0 + tok) * heads + hq];
                if (lse == -INFINITY) seen.lo = seen.hi = 0;
            }
            if (!__any(seen.lo < x.pos + 32 && seen.hi > x.pos)) continue;
            const bool whole = __all(seen.lo <= x.pos && seen.hi >= x.pos + 32);
            u4v q[D / 16];
            const uint16_t *const src = a.q + (s.t0 + tok) * a.q_token + hq * a.q_head + half * (D / 2);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                q[i] = u4v{0, 0, 0, 0};
                if (row < rows) q[i] = *reinterpret_cast<const u4v *>(src + i * 8);
            }
            f16v z;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) z = mfma32<FP16>(k[i], q[i], z);
            const int y0 = x.pos + 4 * half;             // score i is position y0 + 8 (i / 4) + i % 4
            float scale = a.scale_log2;
            if (changed) {
                if (a.cap_log2 > 0.f) {
                    kv_cap<16>(z, a.scale_cap, a.cap_log2);
                    scale = 1.f;
                }
                if (a.slopes && row < rows) {
                    const float slope = a.slopes[hq] * kLog2e, far = (float)(seen.at - y0);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        z[i] = __builtin_fmaf(-slope, fabsf(far - (float)(8 * (i / 4) + i % 4)), z[i] * scale);
                    scale = 1.f;
                }
            }
            const float base = lse * kLog2e;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], scale, -base));
                const int at = y0 + 8 * (i / 4) + i % 4;
                sum[i] += whole || (at >= seen.lo && at < seen.hi) ? e : 0.f;
            }
        }
        // Over the lanes of a half, halving what each holds: in the end the even lanes have
        // position 16 bit 4 + 8 bit 3 + 2 bit 2 + bit 1 of theirs (of a sum's place i).
        int place = 0;
#pragma unroll
        for (int n = 8, m = 16; n >= 1; n /= 2, m /= 2) {
            const bool up = lane & m;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float mine = up ? sum[i + n] : sum[i], theirs = up ? sum[i] : sum[i + n];
                sum[i] = mine + __shfl_xor(theirs, m);
            }
            place += up ? n : 0;
        }
        sum[0] += __shfl_xor(sum[0], 1);
        const int pos = x.pos + 4 * half + 8 * (place / 4) + place % 4;
        if (!(lane & 1) && pos < w.positions) {
            float *const to = w.weights + x.b * w.weights_seq + wrow + pos;
            *to = w.add ? *to + sum[0] : sum[0];
        }
    }
}

template <int D, int SUB>
hipError_t launch(const KvCache &c, const KvNew &a, const KvWeigh &w, hipStream_t s)
{
    const auto kernel = c.fp16 ? kv_weigh_kernel<D, SUB, true> : kv_weigh_kernel<D, SUB, false>;
    const int64_t span = (int64_t)a.table_pages << c.page_log2;
    const int64_t tiles = a.seqs * (((span < w.positions ? span : w.positions) + 31) / 32);
    int64_t splits = 2 * kCUs / c.heads;                 // two workgroups to a CU
    if (splits > (tiles + kWaves - 1) / kWaves) splits = (tiles + kWaves - 1) / kWaves;
    if (splits < 1) splits = 1;
    const size_t lds = Form<D, SUB>::kBook + (a.seqs + 1) * sizeof(int);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(c.heads * splits)), dim3(kThreads), lds, s, c, a, w,
                       (int)splits);
    return hipGetLastError();
}

template <int SUB>
hipError_t launch_sub(const KvCache &c, const KvNew &a, const KvWeigh &w, hipStream_t s)
{
    return c.dim == 64 ? launch<64, SUB>(c, a, w, s)
         : c.dim == 96 ? launch<96, SUB>(c, a, w, s) : launch<128, SUB>(c, a, w, s);
}

}  // namespace

hipError_t launch_kv_weigh(const KvCache &c, const KvNew &a, const KvWeigh &w, hipStream_t s)
{
    return c.sub == 2 ? launch_sub<2>(c, a, w, s) : c.sub == 4 ? launch_sub<4>(c, a, w, s) : launch_sub<8>(c, a, w, s);
}

}  // namespace lloyd
