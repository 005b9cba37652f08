// Eviction: each head of a sequence keeps the positions of the largest weight.
//
// Two launches. The first picks: a workgroup takes a head of a sequence and finds the
// weight that the last kept position has, a byte of its bits after the other by counts of
// the 256 values of each, then writes the kept positions in order. The second moves:
// what goes to place j comes from a position of at least j, so that in place a tile of
// places may be written once all of it, and of the tiles before, has been read.
#include "kv_device.h"
#include "kv_tokens.h"

namespace lloyd {

namespace {

constexpr int kPick = 1024;          // threads that pick
constexpr int kPickWaves = kPick / kWave;
constexpr int kMove = 256;           // threads that move, and places of a tile
constexpr int kParts = 4;            // shares of a token's codes, each moved on its own

// Weights as whole numbers of the same order; NaN below all.
__device__ inline uint32_t order_of(float w)
{
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.f);         // -0 is 0
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ inline int length_of(const KvCache &c, const KvEvict &e, int b)
{
    return min(max(e.lengths[b], 0), e.table_pages << c.page_log2);
}

__global__ __launch_bounds__(kPick) void kv_pick_kernel(KvCache c, KvEvict e)
{
    __shared__ int counts[256];
    __shared__ int found[2];
    __shared__ int wave_gt[kPickWaves], wave_eq[kPickWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x / c.heads, h = blockIdx.x % c.heads;
    const int n = length_of(c, e, b);
    int32_t *const kept = e.kept + ((int64_t)b * c.heads + h) * e.keep;
    if (n <= e.keep) {
        for (int j = tid; j < e.keep; j += kPick) kept[j] = j < n ? j : -1;
        return;
    }
    const float *const w = e.weights + b * e.weights_seq + h * e.weights_head;
    const int from = e.first, to = n - e.recent;         // picked among these
    const auto order_at = [&](int i) { return i < e.positions ? order_of(w[i]) : order_of(0.f); };
    int left = e.keep - e.first - e.recent;              // still to be picked
    uint32_t last = 0, mask = 0;                         // the bits known of the last one
    for (int j = tid; j < e.first; j += kPick) kept[j] = j;
    for (int j = tid; j < e.recent; j += kPick) kept[e.keep - e.recent + j] = to + j;
    if (left == 0) return;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) counts[tid] = 0;
        __syncthreads();
        for (int i = from + tid; i < to; i += kPick) {
            const uint32_t u = order_at(i);
            if ((u & mask) == last) atomicAdd(&counts[u >> shift & 255], 1);
        }
        __syncthreads();
        if (wave == 0) {
            // bins 4 lane to 4 lane + 3, and how many lie in the lanes above
            const int4 n4 = reinterpret_cast<const int4 *>(counts)[lane];
            int above = n4.x + n4.y + n4.z + n4.w;
            const int own = above;
            for (int k = 1; k < kWave; k *= 2) {
                const int x = __shfl_down(above, k);
                if (lane + k < kWave) above += x;
            }
            above -= own;
            const int bins[4] = {n4.x, n4.y, n4.z, n4.w};
            for (int k = 3; k >= 0; --k) {
                if (above < left && above + bins[k] >= left) {
                    found[0] = 4 * lane + k;
                    found[1] = left - above;
                }
                above += bins[k];
            }
        }
        __syncthreads();
        last |= (uint32_t)found[0] << shift;
        mask |= 255u << shift;
        left = found[1];
        __syncthreads();
    }
    // All above `last`, and the first `left` of those alike.
    const int each = ((to - from + kPick - 1) / kPick) * kWave;
    const int w0 = min(from + wave * each, to), w1 = min(w0 + each, to);
    int gt = 0, eq = 0;
    for (int i = w0; i < w1; i += kWave) {
        const uint32_t u = i + lane < w1 ? order_at(i + lane) : 0;
        gt += __popcll(__ballot(i + lane < w1 && u > last));
        eq += __popcll(__ballot(i + lane < w1 && u == last));
    }
    if (lane == 0) {
        wave_gt[wave] = gt;
        wave_eq[wave] = eq;
    }
    __syncthreads();
    int alike = 0, at = e.first;
    for (int k = 0; k < wave; ++k) {
        at += wave_gt[k];
        alike += wave_eq[k];
    }
    at += min(alike, left);
    for (int i = w0; i < w1; i += kWave) {
        const uint32_t u = i + lane < w1 ? order_at(i + lane) : 0;
        const uint64_t below = (1ull << lane) - 1;
        const uint64_t same = __ballot(i + lane < w1 && u == last);
        const bool take = i + lane < w1 &&
                          (u > last || (u == last && alike + __popcll(same & below) < left));
        const uint64_t taken = __ballot(take);
        if (take) kept[at + __popcll(taken & below)] = i + lane;
        at += __popcll(taken);
        alike += __popcll(same);
    }
}

// Part 0: the weights; 1 to kParts: keys' codes; then the values'. A workgroup takes
// every step-th tile of its part, in place all of them.
template <int S>
__global__ __launch_bounds__(kMove) void kv_move_kernel(KvCache c, KvEvict e, int tiles, int step)
{
    constexpr int words = (S / 4 + kParts - 1) / kParts; // of a key's codes, to a part
    constexpr int subs = (S + kParts - 1) / kParts;      // of a value's
    constexpr int runs = (kMove / 8 * subs + kMove - 1) / kMove;
    __shared__ int32_t s_page[kMove];
    __shared__ int32_t s_off[kMove];
    const int tid = threadIdx.x;
    const int part = blockIdx.x % (2 * kParts + 1), bh = blockIdx.x / (2 * kParts + 1) % (c.heads * e.seqs);
    const int tile0 = blockIdx.x / (2 * kParts + 1) / (c.heads * e.seqs);
    const int b = bh / c.heads, h = bh % c.heads;
    const int m = min(length_of(c, e, b), e.keep);
    const int32_t *const kept = e.kept + (int64_t)bh * e.keep;
    if (part == 0) {
        const float *const in = e.weights + b * e.weights_seq + h * e.weights_head;
        float *const out = e.weights_out + b * e.out_seq + h * e.out_head;
        for (int tile = tile0; tile < tiles; tile += step) {
            const int64_t j = (int64_t)tile * kMove + tid;
            float x = 0.f;
            if (j < m) {
                const int i = kept[j];
                if (i < e.positions) x = in[i];
            }
            __syncthreads();
            if (j < e.positions) out[j] = x;
        }
        if (tile0 == 0 && h == 0 && tid == 0) e.lengths_out[b] = m;
        return;
    }
    if (m == 0 || (e.in_place && kept[m - 1] == m - 1)) return;      // all where they are
    const uint32_t last = (uint32_t)min(c.pages - 1, (int64_t)0x7FFFFFFF);
    const int mask = (1 << c.page_log2) - 1;
    const int32_t *const table = e.table + b * e.table_stride, *const to = e.to + b * e.to_stride;
    for (int tile = tile0; tile < tiles && tile * kMove < m; tile += step) {
        const int j0 = tile * kMove;
        __syncthreads();
        if (j0 + tid < m) {
            const int i = kept[j0 + tid];
            s_page[tid] = (int)min((uint32_t)table[i >> c.page_log2], last);
            s_off[tid] = i & mask;
        }
        __syncthreads();
        if (part <= kParts) {
            const int w0 = (part - 1) * words;
            const int j = j0 + tid;
            uint32_t x[words];
            if (j < m) {
                const uint8_t *src = c.k_codes + kv_head(c, s_page[tid], h, S) + (int64_t)s_off[tid] * S;
#pragma unroll
                for (int k = 0; k < words; ++k)
                    if (w0 + k < S / 4) x[k] = reinterpret_cast<const uint32_t *>(src)[w0 + k];
            }
            if (e.in_place) __syncthreads();
            if (j < m) {
                const uint32_t page = (uint32_t)to[j >> c.page_log2];
                if (page <= last) {
                    uint8_t *dst = c.k_codes + kv_head(c, page, h, S) + (int64_t)(j & mask) * S;
#pragma unroll
                    for (int k = 0; k < words; ++k)
                        if (w0 + k < S / 4) reinterpret_cast<uint32_t *>(dst)[w0 + k] = x[k];
                }
            }
        } else {
            const int s0 = (part - 1 - kParts) * subs;
            uint64_t x[runs];
#pragma unroll
            for (int k = 0; k < runs; ++k) {
                const int u = k * kMove + tid, sub = s0 + u / (kMove / 8), g = u % (kMove / 8) * 8;
                x[k] = 0;
                if (u >= kMove / 8 * subs || sub >= S || j0 + g >= m) continue;
#pragma unroll
                for (int y = 0; y < 8; ++y)
                    if (j0 + g + y < m)
                        x[k] |= (uint64_t)c.v_codes[kv_head(c, s_page[g + y], h, S) +
                                                    ((int64_t)sub << c.page_log2) + s_off[g + y]]
                                << (8 * y);
            }
            if (e.in_place) __syncthreads();
#pragma unroll
            for (int k = 0; k < runs; ++k) {
                const int u = k * kMove + tid, sub = s0 + u / (kMove / 8), g = u % (kMove / 8) * 8;
                const int j = j0 + g;
                if (u >= kMove / 8 * subs || sub >= S || j >= m) continue;
                const uint32_t page = (uint32_t)to[j >> c.page_log2];
                if (page > last) continue;
                uint8_t *dst = c.v_codes + kv_head(c, page, h, S) + ((int64_t)sub << c.page_log2) + (j & mask);
                if (j + 8 <= m)
                    *reinterpret_cast<uint64_t *>(dst) = x[k];
                else
                    for (int y = 0; y < m - j; ++y) dst[y] = (uint8_t)(x[k] >> (8 * y));
            }
        }
    }
}

template <int S>
void move(const KvCache &c, const KvEvict &e, hipStream_t s)
{
    // places that any sequence can have, and those of a row of weights
    int64_t most = (int64_t)e.table_pages << c.page_log2;
    if (most > e.keep) most = e.keep;
    if (most < e.positions) most = e.positions;
    const int tiles = (int)((most + kMove - 1) / kMove);
    const int64_t rows = (int64_t)c.heads * e.seqs * (2 * kParts + 1);
    // out of place a workgroup to a tile, up to some 2^22 of them
    int64_t step = e.in_place ? 1 : ((int64_t)1 << 22) / rows;
    step = step < 1 ? 1 : step > tiles ? tiles : step;
    hipLaunchKernelGGL((kv_move_kernel<S>), dim3((unsigned)(rows * step)), dim3(kMove), 0, s, c, e,
                       tiles, (int)step);
}

}  // namespace

hipError_t launch_kv_evict(const KvCache &c, const KvEvict &e, hipStream_t s)
{
    hipLaunchKernelGGL(kv_pick_kernel, dim3((unsigned)(c.heads * e.seqs)), dim3(kPick), 0, s, c, e);
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
    switch (c.dim / c.sub) {
    case 8: move<8>(c, e, s); break;
    case 12: move<12>(c, e, s); break;
    case 16: move<16>(c, e, s); break;
    case 24: move<24>(c, e, s); break;
    case 32: move<32>(c, e, s); break;
    case 48: move<48>(c, e, s); break;
    default: move<64>(c, e, s); break;
    }
    return hipGetLastError();
}

}  // namespace lloyd
