// The weight that attention gave to cached positions.
//
// A wave takes a tile of 32 positions of a sequence, looks their keys up once from the
// centres of its head in LDS, which become the rows of one operand of
// v_mfma_f32_32x32x16, and goes through the rows of the sequence's new tokens (the query
// heads of each), 32 at a time as columns of the other: exp(z - lse) is summed for each
// position in its lanes, and over the lanes at the end. Where positions are few and rows many
// the waves of a workgroup share a tile's rows and add up over LDS. Each sum has one order
// and one writer.
//
// The keys' codes are the bytes that must come from memory. For a single new token it is their
// way that takes the time, and what a launch takes before its first tile (some 9 us: the
// centres to LDS, behind them the first page numbers, codes and rows, one after the other): 32
// sequences of 512 to 4096, 4 heads to each of 8 key heads of 128, bf16, 19.7 us.
// For many the vector ALU does, with 19 operations to a score under a cap, 9 without, and the
// way that tiles fall to waves (some 3 to one): the last 33 to 64 tokens of 4 prompts of 5000
// to 8000, 8 heads to a key head, capped, 82 to 85 us, 0.25 PFLOP/s of products. Tiles before
// what a window shows are left out; those that starts hide are worked on and weigh nothing.
#include "kv_tokens_device.h"

#include <type_traits>

namespace lloyd {

namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
// Tiles whose codes are under way to a wave: with four 32 sequences of 4096 took 18.5 us, with
// one 20.4; more would not fit the registers.
constexpr int kAhead = 4;
constexpr int kSeqs = 512;           // sequences that are kept in LDS

template <int D, int SUB>
struct Form {
    static constexpr int S = D / SUB, H = S / 2;         // codes of a key, of a lane's half of it
    static constexpr int kBook = D * 512;                // [S][256][SUB]
    static constexpr int kRow = D * 2 + 16;              // bytes of a row of queries in LDS: rows that
    static constexpr int kRows = kWaves * 32 * kRow;     // lanes read at once begin on banks of their own
    static constexpr size_t lds(int64_t sequences)
    {
        return kBook + kRows + kSeqs * sizeof(KvSeq) + 2 * kWaves * 32 * sizeof(float) +
               (kWaves + sequences + 1) * sizeof(unsigned);
    }
    static_assert(kBook + kRows + kSeqs * sizeof(KvSeq) + 2 * kWaves * 32 * sizeof(float) +
                  (kWaves + kKvMaxSeqs + 1) * sizeof(unsigned) <= kMaxLds, "a workgroup");
};

// N bytes of codes, in whole words.
template <int N>
__device__ inline void load_codes(uint32_t (&dst)[(N + 3) / 4], const uint8_t *src)
{
    constexpr int align = N % 16 == 0 ? 16 : N % 8 == 0 ? 8 : N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1;
    dst[(N - 1) / 4] = 0;
    __builtin_memcpy(dst, __builtin_assume_aligned(src, align), N);
}

// base + code n times the size of an entry; base has no bits below 256 entries.
template <int SUB>
__device__ inline uint32_t code_at(const uint32_t *w, int n, uint32_t base)
{
    constexpr int shift = SUB == 2 ? 2 : SUB == 4 ? 3 : 4;
    const int low = 8 * (n & 3);
    const uint32_t at = low < shift ? w[n >> 2] << (shift - low) : w[n >> 2] >> (low - shift);
    return (at & (255u << shift)) | base;
}

// x of another lane of the row of 16.
template <int DPP>
__device__ inline float moved(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), DPP, 0xF, 0xF, true));
}

// The lanes of which `up` holds keep sums N to 2 N - 1, the others the first N, and get
// what the lane that DPP names has of them.
template <int N, int DPP>
__device__ inline void fold(float (&sum)[16], bool up)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float mine = up ? sum[i + N] : sum[i], theirs = up ? sum[i] : sum[i + N];
        sum[i] = mine + moved<DPP>(theirs);
    }
}

template <int D, int SUB, bool FP16>
__global__ __launch_bounds__(kThreads) void kv_weigh_kernel(KvCache c, KvNew a, KvWeigh w, int splits, int team)
{
    using F = Form<D, SUB>;
    extern __shared__ uint4 lds[];
    // the kernel has no LDS but its dynamic one, which so begins at 0
    char *const book = reinterpret_cast<char *>(lds);
    KvSeq *const seqs = reinterpret_cast<KvSeq *>(book + F::kBook + F::kRows);      // [kSeqs]
    float *const team_sum = reinterpret_cast<float *>(seqs + kSeqs);     // [2][kWaves][32]
    unsigned *const wave_sum = reinterpret_cast<unsigned *>(team_sum + 2 * kWaves * 32);      // [kWaves]
    unsigned *const first = wave_sum + kWaves;                           // [seqs + 1]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int h = blockIdx.x % c.heads, j = blockIdx.x / c.heads;
    const int heads = c.heads * a.group;
    const int64_t wrow = (int64_t)h * w.weights_head;

    // The centres of this head's keys, entries from K up zeros.
    const uint16_t *const from = c.k_centres + (int64_t)h * F::S * c.K * SUB;
    if (c.K == 256) {
#pragma unroll
        for (int i = 0; i < (D * 32 + kThreads - 1) / kThreads; ++i)
            if (i * kThreads + (wave << 6) < D * 32) __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)(reinterpret_cast<const char *>(from) + (i * kThreads + tid) * 16),
                (__attribute__((address_space(3))) void *)(book + (i * kThreads + (wave << 6)) * 16), 16, 0, 0);
    } else {
        for (int i = tid; i < F::S * 256; i += kThreads) {
            KvEntry<SUB> e{};
            if ((i & 255) < c.K) e = kv_load<SUB>(from + ((i >> 8) * c.K + (i & 255)) * SUB);
            reinterpret_cast<KvEntry<SUB> *>(book)[i] = e;
        }
    }
    // A sequence's tiles, and where the work on each one's begins in all of it. One without
    // new tokens has none, and a window leaves out those before it. A tile's work is that
    // of looking its keys up and folding its sums, counted as two blocks of rows, and that of
    // each block.
    const int span = (int)min(w.positions, (int64_t)a.table_pages << c.page_log2);
    const auto tile0_of = [&](const KvSeq &s) {
        return a.window ? max(s.len - s.n - a.window + 1, 0) >> 5 : 0;
    };
    const auto tiles_of = [&](const KvSeq &s) {
        return s.n ? max(((min(s.len, span) + 31) >> 5) - tile0_of(s), 0) : 0;
    };
    const int team_rows = 32 * team, rank = team > 1 ? wave : 0;
    const auto work_of = [&](const KvSeq &s) {
        return 2u + (unsigned)(s.n * a.group + team_rows - 1) / (unsigned)team_rows;
    };
    // (all of it below 2^32: twelve times what the entry point lets be 2^27)
    unsigned all;
    {
        const int per = (a.seqs + kThreads - 1) / kThreads;
        unsigned sum = 0;
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            if (b >= a.seqs) break;
            const KvSeq s = kv_seq(c, a, b);
            sum += (unsigned)tiles_of(s) * work_of(s);
            if (b < kSeqs) seqs[b] = s;
        }
        const unsigned upto = (unsigned)scan_lanes((int)sum);
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        unsigned at = upto - sum;
        all = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            const unsigned x = wave_sum[i];
            at += i < wave ? x : 0u;
            all += x;
        }
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            if (b >= a.seqs) break;
            const KvSeq s = per == 1 && b < kSeqs ? seqs[b] : kv_seq(c, a, b);
            first[b] = at;
            at += (unsigned)tiles_of(s) * work_of(s);
        }
        if (tid == 0) first[a.seqs] = all;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the centres
    __syncthreads();
    const auto seq_of = [&](int b) { return b < kSeqs ? seqs[b] : kv_seq(c, a, b); };
    // What no tile covers, for the waves that have done their share.
    const auto clear = [&]() {
        if (w.add) return;
        for (int b = j; b < a.seqs; b += splits) {
            float *const to = w.weights + b * w.weights_seq + wrow;
            const KvSeq s = seq_of(b);
            const int n = tiles_of(s), tile0 = n ? tile0_of(s) : 0;
            for (int i = tid; i < tile0 * 32; i += kThreads) to[i] = 0.f;
            for (int64_t i = (int64_t)(tile0 + n) * 32 + tid; i < w.positions; i += kThreads) to[i] = 0.f;
        }
    };

    const unsigned page_bytes = (unsigned)(c.heads * F::S) << c.page_log2;
    const unsigned last_page = (unsigned)min(c.pages - 1, (int64_t)0x7FFFFFFF);
    const unsigned pm = (1u << c.page_log2) - 1;
    const uint8_t *const lane_codes = c.k_codes + (((int64_t)h * F::S) << c.page_log2) + half * F::H;
    // A wave's share, or that of a team: the tiles whose work begins in an even share of all.
    const unsigned shares = team > 1 ? splits : kWaves * splits, share = team > 1 ? j : j * kWaves + wave;
    all = __builtin_amdgcn_readfirstlane(all);
    const unsigned each = all / shares, over = all - each * shares;
    const unsigned work0 = each * share + min(share, over), work1 = work0 + each + (share < over);
    // A place among the tiles: tile t of sequence b, of which the wave's are those up to
    // `end` of its n.
    struct Place {
        int b, t, end, n, tile0;
        KvSeq s;
        const int32_t *row;
    };
    const auto enter = [&](int b) {
        Place x;
        x.b = __builtin_amdgcn_readfirstlane(b);
        const KvSeq s = seq_of(x.b);
        x.s.t0 = __builtin_amdgcn_readfirstlane(s.t0);
        x.s.n = __builtin_amdgcn_readfirstlane(s.n);
        x.s.len = __builtin_amdgcn_readfirstlane(s.len);
        x.s.prefix = __builtin_amdgcn_readfirstlane(s.prefix);
        x.row = a.table + x.b * a.table_stride;
        x.n = tiles_of(x.s);
        x.tile0 = tile0_of(x.s);
        const unsigned from = __builtin_amdgcn_readfirstlane(first[x.b]), work = work_of(x.s);
        const auto tiles_before = [&](unsigned to) {     // that begin there
            return to <= from ? 0 : to - from >= x.n * work ? x.n : (int)((to - from + work - 1) / work);
        };
        x.t = tiles_before(work0);
        x.end = tiles_before(work1);
        return x;
    };
    // Whether there is a tile at x that is the wave's, or one in a sequence after it.
    const auto settle = [&](Place &x) {
        while (x.t >= x.end) {
            if (x.end < x.n) return false;
            // the next sequence that has tiles: of 64 at a time
            int b = x.b + 1;
            for (;;) {
                const int n = b + lane;
                const uint64_t some = __ballot(n < a.seqs && first[min(n, a.seqs)] < first[min(n + 1, a.seqs)]);
                if (some) {
                    b += __builtin_ctzll(some);
                    break;
                }
                b += kWave;
                if (b >= a.seqs) return false;
            }
            x = enter(b);
        }
        return true;
    };
    // A lane's page of the tile at x.
    struct Where {
        int pos, page;
    };
    const auto find = [&](const Place &x) {
        Where y;
        y.pos = (x.t + x.tile0) * 32;
        y.page = x.row[(unsigned)min(y.pos + col, x.s.len - 1) >> c.page_log2];
        return y;
    };
    const auto load = [&](uint32_t (&codes)[(F::H + 3) / 4], const Where &y) {
        load_codes<F::H>(codes, lane_codes + (uint64_t)min((unsigned)y.page, last_page) * page_bytes +
                                    (((unsigned)y.pos + col) & pm) * F::S);
    };
    if (work0 >= work1) return clear();
    Place now;
    {
        // the sequence in whose tiles work0 lies: the last that begins at it or before
        int b = 0;
        for (;;) {
            const int n = b + 1 + lane;
            const int more = __popcll(__ballot(n < a.seqs && first[min(n, a.seqs)] <= work0));
            b += more;
            if (more < kWave) break;
        }
        now = enter(b);
    }
    if (!settle(now)) return clear();
    // Codes are asked for kAhead tiles before they are looked up, numbers of pages twice as
    // many; behind the last tile, some tile's again.
    Place next = now;
    bool more = true;
    Where where[kAhead]{};
    uint32_t codes[kAhead][(F::H + 3) / 4];
    const auto find_next = [&](Where &x) {
        if (!more) return;
        x = find(next);
        ++next.t;
        more = settle(next);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        if (i) where[i] = where[i - 1];
        find_next(where[i]);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(codes[i], where[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) find_next(where[i]);
    // 32 rows: a lane has its token's number in the sequence and start, logarithm and slope of
    // row `col` of them. The queries come from memory 1024 bytes of rows to a load, a block
    // ahead, and go to LDS, where each lane has its half of a row for the products: a block
    // takes some 3600 cycles. Loaded as the products take them, 16 bytes of 64 half rows to a
    // load, it took 5000, half of them waiting for the rows.
    struct Rows {
        int tok, start;
        float lse, slope;
    };
    Rows cur, coming;
    u4v raw[D / 16];                                     // the queries of the coming rows
    const uint32_t wave_rows = F::kBook + wave * (32 * F::kRow);
    int loaded = -1;                                     // the sequence whose rows are in LDS
    int next_row = 0;                                    // the first of those to ask for
    const int tokens_on = team_rows / a.group, heads_on = team_rows % a.group;
    int tok = 0, hd = 0;                                 // of the next block's row
    // the sequence's first rows come next
    const auto rewind = [&]() {
        next_row = 32 * rank;
        tok = (int)((unsigned)(32 * rank + col) / (unsigned)a.group);
        hd = (int)((unsigned)(32 * rank + col) % (unsigned)a.group);
    };
    const auto begin = [&](const KvSeq &s) {
        Rows &x = coming;
        // behind the last row: some row
        const int64_t t = s.t0 + min(tok, s.n - 1);
        const int hq = h * a.group + hd;
        x.tok = tok;
        x.start = a.starts ? a.starts[t] : 0;
        x.lse = w.lse[t * heads + hq];
        x.slope = a.slopes ? a.slopes[hq] : 0.f;
        const uint64_t src = reinterpret_cast<uint64_t>(a.q + t * a.q_token + hq * a.q_head);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const int row = (i * kWave + lane) / (D / 8), chunk = (i * kWave + lane) % (D / 8);
            const uint32_t lo = __builtin_amdgcn_ds_bpermute(row * 4, (int)(uint32_t)src);
            const uint32_t hi = __builtin_amdgcn_ds_bpermute(row * 4, (int)(uint32_t)(src >> 32));
            raw[i] = *(const __attribute__((address_space(1))) u4v *)(((uint64_t)hi << 32 | lo) + chunk * 16);
        }
        tok += tokens_on;
        hd += heads_on;
        if (hd >= a.group) {
            hd -= a.group;
            ++tok;
        }
        next_row += team_rows;
        if (next_row >= s.n * a.group) rewind();         // behind the last: the first, for the next tile
    };
    // The rows that begin() asked for are the ones at hand.
    const auto take = [&]() {
        cur = coming;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            lds_put(wave_rows + (i * kWave + lane) / (D / 8) * F::kRow + (i * kWave + lane) % (D / 8) * 16, 0, raw[i]);
        asm volatile("" ::: "memory");                   // a wave's LDS accesses keep their order
    };
    // The tile at `now`, whose codes are codes[I]. False: it was the last.
    const auto turn = [&](auto I) {
        constexpr int slot = decltype(I)::value;
        // the keys: a lane has features [half D / 2, + D / 2) of position col
        u4v k[D / 16];
        {
            KvEntry<SUB> e[F::H];
#pragma unroll
            for (int n = 0; n < F::H; ++n)
                e[n] = lds_get<KvEntry<SUB>>(code_at<SUB>(codes[slot], n, half * (F::H * 512 * SUB)), n * (512 * SUB));
            __builtin_memcpy(k, e, sizeof(k));
        }
        load(codes[slot], where[slot]);
        find_next(where[slot]);
        const int b = now.b, pos = (now.t + now.tile0) * 32;
        const KvSeq s = now.s;
        float sum[16] = {};
        const int rows = s.n * a.group;
        if (loaded != b) {
            loaded = b;
            rewind();
            begin(s);
            __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0), or the compiler waits below,
            take();                                      // where codes are under way
            if (rows > team_rows) begin(s);
        }
#pragma unroll 1
        for (int r0 = 32 * rank;; r0 += team_rows) {
            const Rows x = cur;
            KvSeen seen = kv_seen(a, s, x.tok, x.start);
            const float base = x.lse * kLog2e;
            if (x.tok >= s.n || base == -INFINITY) seen.lo = seen.hi = 0;
            const bool any = __any(seen.lo < pos + 32 && seen.hi > pos);
            const bool whole = __ballot(seen.lo <= pos && seen.hi >= pos + 32) == ~0ull;
            f16v z;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.f;
            if (any) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
                    z = mfma32<FP16>(k[i], lds_get<u4v>(wave_rows + col * F::kRow + half * D, i * 16), z);
                asm volatile("" ::: "memory");
            }
            if (rows > team_rows) {
                take();
                begin(s);
            }
            if (any) {
                const int y0 = pos + 4 * half;               // score i is position y0 + 8 (i / 4) + i % 4
                if (a.cap_log2 > 0.f) kv_cap<16>(z, a);
                const float scale = a.cap_log2 > 0.f ? 1.f : a.scale_log2;
                if (a.slopes) {
                    const float far = (float)(seen.at - y0), slope = x.slope * kLog2e;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        z[i] = __builtin_fmaf(-slope, fabsf(far - (float)(8 * (i / 4) + i % 4)), z[i] * scale) - base;
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = __builtin_fmaf(z[i], scale, -base);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = __builtin_amdgcn_exp2f(z[i]);
                if (whole) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[i] += z[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int p = y0 + 8 * (i / 4) + i % 4;
                        sum[i] += p >= seen.lo && p < seen.hi ? z[i] : 0.f;
                    }
                }
            }
            if (r0 + team_rows >= rows) break;
        }
        // Over the 32 lanes of a half, halving what each holds (rows of 16 exchange, then
        // lanes 8, 7, 2 and 1 away): place i of the sums in the end is 8 bit 4 + 4 bit 3 +
        // 2 bit 2 + bit 1 of the lane.
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum[i]), __float_as_uint(sum[i + 8]), false, false);
            sum[i] = __uint_as_float(both[0]) + __uint_as_float(both[1]);
        }
        fold<4, 0x128>(sum, lane & 8);                   // row_ror:8
        fold<2, 0x141>(sum, lane & 4);                   // row_half_mirror
        fold<1, 0x4E>(sum, lane & 2);                    // quad_perm:[2,3,0,1]
        sum[0] += moved<0xB1>(sum[0]);                   // quad_perm:[1,0,3,2]
        const int place = (lane & 16) / 2 + (lane & 8) / 2 + (lane & 4) / 2 + (lane & 2) / 2;
        int at = 4 * half + 8 * (place / 4) + place % 4;
        bool mine = !(lane & 1);
        if (team > 1) {
            // (two of them: the first wave reads a tile's while the others write the next)
            float *const to = team_sum + slot % 2 * (kWaves * 32);
            if (mine) to[wave * 32 + at] = sum[0];
            lds_barrier();
            at = col;
            mine = wave == 0 && half == 0;
            if (mine) {
                sum[0] = to[at];
#pragma unroll
                for (int i = 1; i < kWaves; ++i) sum[0] += to[i * 32 + at];
            }
        }
        if (mine && pos + at < w.positions) {
            float *const to = w.weights + b * w.weights_seq + wrow + pos + at;
            *to = w.add ? *to + sum[0] : sum[0];
        }
        ++now.t;
        return settle(now);
    };
    while (turn(std::integral_constant<int, 0>{}) && turn(std::integral_constant<int, 1>{}) &&
           turn(std::integral_constant<int, 2>{}) && turn(std::integral_constant<int, 3>{})) {}
    clear();
}

template <int D, int SUB>
hipError_t launch(const KvCache &c, const KvNew &a, const KvWeigh &w, hipStream_t s)
{
    const auto kernel = c.fp16 ? kv_weigh_kernel<D, SUB, true> : kv_weigh_kernel<D, SUB, false>;
    const int64_t span = (int64_t)a.table_pages << c.page_log2;
    const int64_t tiles = a.seqs * (((span < w.positions ? span : w.positions) + 31) / 32);
    const auto over = [](int64_t n, int64_t k) { return (n + k - 1) / k; };
    const auto splits_of = [&](int64_t n) {
        const int64_t most = kCUs / c.heads;
        return n > most ? (most < 1 ? 1 : most) : n < 1 ? 1 : n;
    };
    // A tile to a wave, or, of few positions and many rows, to all waves of a workgroup, its
    // rows shared: what takes less work, were all sequences as long as the table's rows. In us,
    // alone and shared, 8 heads of 128, bf16: 47 and 71 (4 sequences of 5000, 33 tokens of 8
    // heads), 92 and 121 (of 8000, 64 tokens), 20 and 32 (of 2000, 33 tokens), 27 and 24 (of 1000,
    // 128 tokens of 4), 48 and 25 (one of 2000, 256 tokens), 18 and 11 (64 tokens); of one head of
    // 300 positions, 1000 tokens of 8, 313 and 46. Where the rule gives both about the same: 38 and
    // 36 (8 of 2000, 64 tokens of 4: alone), 25 and 26 (4 heads, 3 of 3000, 100 tokens of 4: shared).
    const int64_t alone = splits_of(over(tiles, kWaves)), together = splits_of(tiles);
    const int64_t blocks = over(over(a.tokens * a.group, a.seqs), 32);
    const bool team = over(tiles, together) * (1 + 2 * over(blocks, kWaves)) < over(tiles, alone * kWaves) * (1 + 2 * blocks);
    const int64_t splits = team ? together : alone;
    const size_t lds = Form<D, SUB>::lds(a.seqs);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(c.heads * splits)), dim3(kThreads), lds, s, c, a, w,
                       (int)splits, team ? kWaves : 1);
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
