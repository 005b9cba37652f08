// Eviction: each head of a sequence keeps the positions of the largest weight.
//
// Two launches. The first picks: a workgroup takes a head of a sequence, holds its weights in
// registers as whole numbers of the same order, and finds the weight that the last kept
// position has, 11, 11 and 10 of its bits after the other by counts of their values, then
// writes the kept positions in order. The second moves: what goes to place j comes from a
// position of at least j, so that in place a tile of places may be written once all of it,
// and of the tiles before, has been read.
//
// Nothing is computed: bytes bound it, and for short contexts the two launches. 64 contexts
// of 5000 to 8192 positions brought to 4096, 8 heads of 128 in 32 + 32 bytes: the pick 22 us
// (13 MB of weights, three passes over them in registers), the move 88 us, 375 MB read and
// written at 4.3 TB/s, of which keys alone run at 6.4 TB/s and values, gathered by bytes, at 3.4.
// Both launches, us, all contexts of 8192 and codes not in a cache: 150 brought to a half and 111 to
// a tenth (which gathers values by single bytes); in place, where a row has six workgroups that
// take its tiles one after the other, 233 and 135. One context of 65536: 114 and 103, in place 327
// and 170.
#include "kv_tokens_device.h"

namespace lloyd {

namespace {

// Threads that pick, of a row's positions up to kLong and beyond (as many as the table has room
// for). In us, with 512 and 1024, and the move after it: 72 and 79 (64 sequences of 8192, 8
// heads), 22 and 20 (4 of 8192), 36 and 30 (4 of 16000), 80 and 71 (32 of 16000), 174 and 76 (one
// of 65536), 271 and 152 (4 of 100000).
constexpr int kUsual = 512, kMost = 1024, kLong = 8192;
constexpr int kMove = 256;           // threads that move
// Positions between a tile's first and last that LDS holds. Half of 8192 kept, a tile of 256
// places spans some 512: with 512 half of the tiles were picked from memory, and the values
// took 56 us instead of 51.
constexpr int kSpan = 768;
constexpr int kParts = 4;            // shares of a value's codes, in place each moved on its own

// Weights as whole numbers of the same order; NaN, 1, below all. 0 is no weight's.
__device__ inline uint32_t order_of(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);         // -0 is 0
    return w != w ? 1u : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ inline int length_of(const KvCache &c, const KvEvict &e, int b)
{
    return min(max(e.lengths[b], 0), e.table_pages << c.page_log2);
}

// How many of a row's weights a thread holds at most; longer rows are read again in each pass.
// (26 of 64 go to memory, and 65536 positions take 76 us; read again, 100.)
constexpr int kHeld = 64;
static_assert(kLong <= 16 * kUsual, "all are held");

struct PickLds {
    int counts[2048];
    int wave_sum[16], wave_eq[16];
    int found[2];
};

// The positions [from, to) of a row, wave after wave and in each 64 at a time: f(i, the
// order of its weight), of 64 whole ones that may go beyond `to`, where that is 0.
template <int T, int HELD, typename G, typename F>
__device__ inline void each_of(int from, int to, const uint32_t (&held)[HELD ? HELD : 1], const G &order_at, const F &f)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int each = ((to - from + T - 1) / T) * kWave, w0 = from + wave * each;
    if constexpr (HELD) {
#pragma unroll
        for (int r = 0; r < HELD; ++r) {
            const int i = w0 + r * kWave + lane;
            if (r * kWave < each && w0 + r * kWave < to) f(i, held[r]);
        }
    } else {
        for (int i = w0 + lane; i - lane < min(w0 + each, to); i += kWave) {
            f(i, i < min(w0 + each, to) ? order_at(i) : 0u);
        }
    }
}

// Writes the `left` (at least 1) positions of [from, to) with the largest weights, in order.
template <int T, int HELD, typename G>
__device__ inline void pick(PickLds &lds, int from, int to, int left, int32_t *out, const G &order_at)
{
    constexpr int B = 2048 / T;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t held[HELD ? HELD : 1];
    if constexpr (HELD) {
        const int each = ((to - from + T - 1) / T) * kWave, i0 = from + wave * each + lane;
#pragma unroll
        for (int r = 0; r < HELD; ++r)
            held[r] = r * kWave < each && i0 + r * kWave < to ? order_at(i0 + r * kWave) : 0u;
    }
    uint32_t last = 0, mask = 0;                         // the bits known of the last one
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
        // 11, 11 and 10 bits: the first has an octave's four quarters apart, so that
        // lanes seldom count the same value
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
        const uint32_t bins = digit == 2 ? 1023u : 2047u;
#pragma unroll
        for (int k = 0; k < B; ++k) lds.counts[B * tid + k] = 0;
        __syncthreads();
        each_of<T, HELD>(from, to, held, order_at, [&](int, uint32_t u) {
            // many weights may be alike: what the first lane counts is counted at once for all
            const bool counts = (u & mask) == last;
            const uint64_t some = __ballot(counts);
            if (!some) return;
            const int lead = __builtin_ctzll(some), bin = (int)(u >> shift & bins);
            const int of = __builtin_amdgcn_readlane(bin, lead);
            const uint64_t alike = __ballot(counts && bin == of);
            if (lane == lead) atomicAdd(&lds.counts[of], __popcll(alike));
            if (counts && bin != of) atomicAdd(&lds.counts[bin], 1);
        });
        __syncthreads();
        // thread t has bins B t to B t + B - 1; how many lie above those
        int n[B], own = 0;
#pragma unroll
        for (int k = 0; k < B; ++k) own += n[k] = lds.counts[B * tid + k];
        int above = own;
#pragma unroll
        for (int k = 1; k < kWave; k *= 2) {
            const int x = __shfl_down(above, k);
            if (lane + k < kWave) above += x;
        }
        if (lane == 0) lds.wave_sum[wave] = above;
        __syncthreads();
        above -= own;
#pragma unroll
        for (int k = 1; k < T / kWave; ++k) above += k > wave ? lds.wave_sum[k] : 0;
        if (above < left && above + own >= left) {
#pragma unroll
            for (int k = B - 1; k >= 0; --k) {
                if (above < left && above + n[k] >= left) {
                    lds.found[0] = B * tid + k;
                    lds.found[1] = left - above;
                }
                above += n[k];
            }
        }
        __syncthreads();
        last |= (uint32_t)lds.found[0] << shift;
        mask |= bins << shift;
        left = lds.found[1];
    }
    // All above `last`, and the first `left` of those alike.
    int gt = 0, eq = 0;
    each_of<T, HELD>(from, to, held, order_at, [&](int, uint32_t u) {
        gt += __popcll(__ballot(u > last));
        eq += __popcll(__ballot(u == last));
    });
    if (lane == 0) {
        lds.wave_sum[wave] = gt;
        lds.wave_eq[wave] = eq;
    }
    __syncthreads();
    int alike = 0, at = 0;
#pragma unroll
    for (int k = 0; k < T / kWave - 1; ++k) {
        at += k < wave ? lds.wave_sum[k] : 0;
        alike += k < wave ? lds.wave_eq[k] : 0;
    }
    at += min(alike, left);
    const uint64_t below = (1ull << lane) - 1;
    each_of<T, HELD>(from, to, held, order_at, [&](int i, uint32_t u) {
        const uint64_t same = __ballot(u == last);
        const bool take = u > last || (u == last && alike + __popcll(same & below) < left);
        const uint64_t taken = __ballot(take);
        if (take) out[at + __popcll(taken & below)] = i;
        at += __popcll(taken);
        alike += __popcll(same);
    });
}

template <int T>
__global__ __launch_bounds__(T) void kv_pick_kernel(KvCache c, KvEvict e)
{
    __shared__ PickLds lds;
    const int tid = threadIdx.x;
    const int b = blockIdx.x / c.heads, h = blockIdx.x % c.heads;
    const int n = length_of(c, e, b);
    int32_t *const kept = e.kept + ((int64_t)b * c.heads + h) * e.keep;
    if (n <= e.keep) {
        for (int j = tid; j < e.keep; j += T) kept[j] = j < n ? j : -1;
        return;
    }
    const float *const w = e.weights + b * e.weights_seq + h * e.weights_head;
    const auto order_at = [&](int i) { return i < e.positions ? order_of(w[i]) : order_of(0.f); };
    const int from = e.first, to = n - e.recent, left = e.keep - e.first - e.recent;
    for (int j = tid; j < e.first; j += T) kept[j] = j;
    for (int j = tid; j < e.recent; j += T) kept[e.keep - e.recent + j] = to + j;
    if (left == 0) return;
    if (to - from <= 4 * T)
        pick<T, 4>(lds, from, to, left, kept + e.first, order_at);
    else if (T == kUsual || to - from <= 16 * T)
        pick<T, 16>(lds, from, to, left, kept + e.first, order_at);
    else if constexpr (T == kMost) {
        if (to - from <= kHeld * T)
            pick<T, kHeld>(lds, from, to, left, kept + e.first, order_at);
        else
            pick<T, 0>(lds, from, to, left, kept + e.first, order_at);
    }
}

// What a workgroup moves: weights, keys' codes or values' codes of a head of a sequence; out
// of place one tile of places, in place all tiles one after the other (of a share of the
// sub-vectors, for values). Weights may be moved in place while codes go to other pages,
// and the other way about. Each thread asks for all that it moves of a tile before it
// waits: the way from a kept position over the table to the codes is three trips to
// memory, and bytes under way are what the card's rate takes.
struct MoveGrid {
    int weights, keys, values;       // workgroups of a row
    __host__ __device__ int all() const { return weights + keys + values; }
};

template <int S>
constexpr int kRun = S % 16 == 0 ? 16 : S % 8 == 0 ? 8 : 4;      // bytes of a key's codes to a thread
constexpr int kHold = 8;             // weights, or runs, of a thread
constexpr int kFloats = kMove * kHold;                           // places of a tile of weights
template <int S>
constexpr int kKeys = kMove * kHold / (S / kRun<S>);             // of keys
constexpr int kValues = 256;                                     // of values
// Workgroups of a CU that move values, each of them tile after tile with the next one's places
// ahead: with 2, 4 and 6 the move took 86, 88 and 89 us, with one to every tile 100.
constexpr int kResident = 4;

template <int N>
struct BytesOf {
    typedef uint32_t type __attribute__((ext_vector_type(N / 4)));
};
template <>
struct BytesOf<4> {
    typedef uint32_t type;
};
template <int N>
using Bytes = typename BytesOf<N>::type;

typedef uint32_t Four __attribute__((ext_vector_type(4)));

// Byte y of word n to byte n of word y.
__device__ inline Four turned(Four a)
{
    const uint32_t b0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400), b1 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400);
    const uint32_t b2 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602), b3 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602);
    return Four{__builtin_amdgcn_perm(b1, b0, 0x05040100), __builtin_amdgcn_perm(b1, b0, 0x07060302),
                __builtin_amdgcn_perm(b3, b2, 0x05040100), __builtin_amdgcn_perm(b3, b2, 0x07060302)};
}

template <int S, bool IN_PLACE>
__global__ __launch_bounds__(kMove) void kv_move_kernel(KvCache c, KvEvict e, MoveGrid grid)
{
    const int tid = threadIdx.x, rows = c.heads * e.seqs;
    const int bh = blockIdx.x % rows, b = bh / c.heads, h = bh % c.heads;
    int part = blockIdx.x / rows;
    const int m = min(length_of(c, e, b), e.keep);
    const int32_t *const kept = e.kept + (int64_t)bh * e.keep;
    const uint32_t last = (uint32_t)min(c.pages - 1, (int64_t)0x7FFFFFFF);
    const int mask = (1 << c.page_log2) - 1;
    const int32_t *const table = e.table + b * e.table_stride, *const to = e.to + b * e.to_stride;
    // values, whose workgroups take longest, come first
    if (part >= grid.values + grid.keys) {
        part -= grid.values + grid.keys;
        const float *const in = e.weights + b * e.weights_seq + h * e.weights_head;
        float *const out = e.weights_out + b * e.out_seq + h * e.out_head;
        if (part == 0 && h == 0 && tid == 0) e.lengths_out[b] = m;
        for (int64_t j0 = (int64_t)part * kFloats + tid; j0 - tid < e.positions; j0 += (int64_t)grid.weights * kFloats) {
            int i[kHold];
            float x[kHold];
#pragma unroll
            for (int k = 0; k < kHold; ++k) i[k] = m ? kept[min(j0 + k * kMove, (int64_t)m - 1)] : 0;
#pragma unroll
            for (int k = 0; k < kHold; ++k) x[k] = in[min((int64_t)i[k], e.positions - 1)];
#pragma unroll
            for (int k = 0; k < kHold; ++k)
                if (j0 + k * kMove >= m || i[k] >= e.positions) x[k] = 0.f;
            if (e.weights_in_place) __syncthreads();
#pragma unroll
            for (int k = 0; k < kHold; ++k)
                if (j0 + k * kMove < e.positions) out[j0 + k * kMove] = x[k];
        }
        return;
    }
    if (m == 0 || (IN_PLACE && kept[m - 1] == m - 1)) return;        // all where they are
    if (part >= grid.values) {
        part -= grid.values;
        constexpr int runs = S / kRun<S>;
        for (int j0 = part * kKeys<S>; j0 < m; j0 += grid.keys * kKeys<S>) {
            int i[kHold], goal[kHold], page[kHold];
            Bytes<kRun<S>> x[kHold];
#pragma unroll
            for (int k = 0; k < kHold; ++k) {
                const int j = min(j0 + (k * kMove + tid) / runs, m - 1);
                i[k] = kept[j];
                goal[k] = to[j >> c.page_log2];
            }
#pragma unroll
            for (int k = 0; k < kHold; ++k) page[k] = table[i[k] >> c.page_log2];
#pragma unroll
            for (int k = 0; k < kHold; ++k)
                x[k] = *reinterpret_cast<const Bytes<kRun<S>> *>(
                    c.k_codes + kv_head(c, min((uint32_t)page[k], last), h, S) + (i[k] & mask) * S +
                    (k * kMove + tid) % runs * kRun<S>);
            if (IN_PLACE) __syncthreads();
#pragma unroll
            for (int k = 0; k < kHold; ++k) {
                const int j = j0 + (k * kMove + tid) / runs;
                if (j < m && (uint32_t)goal[k] <= last)
                    *reinterpret_cast<Bytes<kRun<S>> *>(c.k_codes + kv_head(c, goal[k], h, S) + (j & mask) * S +
                                                        (k * kMove + tid) % runs * kRun<S>) = x[k];
            }
        }
        return;
    }
    // Values: what lies between the tile's first and last position comes to LDS, a thread's
    // 8 positions of 4 sub-vectors at a time, laid out anew as one word to a position, and
    // is picked there by words, which are laid out back. Where little is kept it comes from
    // memory by single bytes.
    constexpr int groups = S / 4, shares = IN_PLACE ? kParts : 1, most = (groups + shares - 1) / shares;
    constexpr int wide = 32, high = kMove / wide;        // a thread's positions and groups: every 32nd 8 and 8th
    constexpr int words = kSpan / 8 / wide, turns = (most + high - 1) / high;
    constexpr int row = kSpan + 4;                       // words of a group's in LDS
    __shared__ __attribute__((aligned(16))) uint32_t s_codes[most * row];
    const int g0 = IN_PLACE ? part * most : 0, g1 = min(g0 + most, groups);
    if (g0 >= g1) return;
    // a wave has 64 positions of all groups: what it asks for at once lies on few pages
    const int lane = tid / kWave * 8 + tid % 8, mine = g0 + tid / 8 % high;
    // A tile at place j0: what the thread keeps of it, where it goes, and between which
    // positions all lie. The next tile's is asked for while this one's codes are under way.
    struct Tile {
        int at[8], i0, end;
        uint32_t goal, page[words];
    };
    const auto find = [&](Tile &x, int j0) {
        const int j = j0 + lane * 8;
        if (j + 8 <= m) {
            __builtin_memcpy(x.at, kept + j, sizeof(x.at));
        } else {
#pragma unroll
            for (int y = 0; y < 8; ++y) x.at[y] = kept[min(j + y, m - 1)];
        }
        x.goal = j < m ? (uint32_t)to[j >> c.page_log2] : ~0u;
        x.i0 = kept[j0] & ~7;
        x.end = kept[min(j0 + kValues, m) - 1] + 1;
    };
    const auto find_pages = [&](Tile &x) {
#pragma unroll
        for (int k = 0; k < words; ++k)
            x.page[k] = min((uint32_t)table[min(x.i0 + (lane + k * wide) * 8, x.end - 1) >> c.page_log2], last);
    };
    const int step = (IN_PLACE ? 1 : grid.values) * kValues;
    int j0 = IN_PLACE ? 0 : part * kValues;
    if (j0 >= m) return;
    Tile now, next;
    find(now, j0);
    find_pages(now);
    for (;;) {
        const int j = j0 + lane * 8;                     // the thread's places
        const int i0 = now.i0, end = now.end, (&at)[8] = now.at;
        const bool more = j0 + step < m;
        Four x[turns][2];                                // of a group: places 0 to 3, 4 to 7
        if (end - i0 <= kSpan) {
            uint64_t w[words][turns][4];
#pragma unroll
            for (int k = 0; k < words; ++k) {
                const int i = min(i0 + (lane + k * wide) * 8, (end - 1) & ~7);
                const uint8_t *const from = c.v_codes + kv_head(c, now.page[k], h, S) + (i & mask);
#pragma unroll
                for (int n = 0; n < turns; ++n)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        w[k][n][y] = *reinterpret_cast<const uint64_t *>(
                            from + ((unsigned)(min(mine + n * high, g1 - 1) + y * groups) << c.page_log2));
            }
            find(next, more ? j0 + step : j0);
#pragma unroll
            for (int k = 0; k < words; ++k)
#pragma unroll
                for (int n = 0; n < turns; ++n) {
                    // (where there is nothing more, what is there again)
                    Four *const dst = reinterpret_cast<Four *>(s_codes + (min(mine + n * high, g1 - 1) - g0) * row + (lane + k * wide) * 8);
                    Four part0, part1;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        part0[y] = (uint32_t)w[k][n][y];
                        part1[y] = (uint32_t)(w[k][n][y] >> 32);
                    }
                    dst[0] = turned(part0);
                    dst[1] = turned(part1);
                }
            lds_barrier();
#pragma unroll
            for (int n = 0; n < turns; ++n) {
                const uint32_t *const from = s_codes + min(mine - g0 + n * high, g1 - g0 - 1) * row - i0;
#pragma unroll
                for (int y = 0; y < 8; ++y) x[n][y / 4][y % 4] = from[at[y]];
                x[n][0] = turned(x[n][0]);
                x[n][1] = turned(x[n][1]);
            }
        } else {
            find(next, more ? j0 + step : j0);
            const uint8_t *from[8];
#pragma unroll
            for (int y = 0; y < 8; ++y)
                from[y] = c.v_codes + kv_head(c, min((uint32_t)table[at[y] >> c.page_log2], last), h, S) + (at[y] & mask);
#pragma unroll
            for (int n = 0; n < turns; ++n)
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const unsigned sub = (unsigned)(min(mine + n * high, g1 - 1) + z * groups) << c.page_log2;
                    uint32_t lo = 0, hi = 0;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        lo |= (uint32_t)from[y][sub] << (8 * y);
                        hi |= (uint32_t)from[y + 4][sub] << (8 * y);
                    }
                    x[n][0][z] = lo;
                    x[n][1][z] = hi;
                }
            if (IN_PLACE) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        find_pages(next);
        lds_barrier();                                   // all read; LDS is done with, too
        if (now.goal <= last) {
            uint8_t *const dst = c.v_codes + kv_head(c, now.goal, h, S) + (j & mask);
#pragma unroll
            for (int n = 0; n < turns; ++n) {
                if (mine + n * high >= g1) continue;
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    uint8_t *const out = dst + ((unsigned)(mine + n * high + z * groups) << c.page_log2);
                    const uint64_t bytes = (uint64_t)x[n][1][z] << 32 | x[n][0][z];
                    if (j + 8 <= m)
                        *reinterpret_cast<uint64_t *>(out) = bytes;
                    else
#pragma unroll 1
                        for (int y = 0; y < m - j; ++y) out[y] = (uint8_t)(bytes >> (8 * y));
                }
            }
        }
        if (!more) break;
        now = next;
        j0 += step;
    }
}

template <int S>
void move(const KvCache &c, const KvEvict &e, hipStream_t s)
{
    const int64_t rows = (int64_t)c.heads * e.seqs;
    MoveGrid grid{1, 1, kParts};
    if (!e.in_place) {
        // a workgroup to a tile, up to some 2^22 in all
        int64_t most = (int64_t)e.table_pages << c.page_log2;
        if (most > e.keep) most = e.keep;
        const int64_t room = ((int64_t)1 << 22) / (3 * rows);
        const auto tiles = [&](int64_t n, int tile) {
            n = (n + tile - 1) / tile;
            return (int)(n > room ? room : n < 1 ? 1 : n);
        };
        grid = MoveGrid{e.weights_in_place ? 1 : tiles(e.positions, kFloats), tiles(most, kKeys<S>),
                        tiles(most, kValues)};
        // of values, no more than are at work at once
        const int64_t values = kResident * kCUs / rows;
        if (grid.values > values) grid.values = (int)(values < 1 ? 1 : values);
    }
    const dim3 blocks((unsigned)(rows * grid.all()));
    if (e.in_place)
        hipLaunchKernelGGL((kv_move_kernel<S, true>), blocks, dim3(kMove), 0, s, c, e, grid);
    else
        hipLaunchKernelGGL((kv_move_kernel<S, false>), blocks, dim3(kMove), 0, s, c, e, grid);
}

}  // namespace

hipError_t launch_kv_evict(const KvCache &c, const KvEvict &e, hipStream_t s)
{
    const dim3 rows((unsigned)(c.heads * e.seqs));
    if ((int64_t)e.table_pages << c.page_log2 > kLong)
        hipLaunchKernelGGL(kv_pick_kernel<kMost>, rows, dim3(kMost), 0, s, c, e);
    else
        hipLaunchKernelGGL(kv_pick_kernel<kUsual>, rows, dim3(kUsual), 0, s, c, e);
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
