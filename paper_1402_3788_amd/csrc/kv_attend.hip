// Attention of one new token of every sequence over the cache of codes.
//
// With the scores z_i = scale (q . k_i) in base 2 and a reference m, one pass over
// the positions keeps sum_i 2^(z_i - m) and sum_i 2^(z_i - m) v_i, both scaled when
// the reference is moved up; parts with references of their own are joined by
// 2^(m - largest m).
//
// A workgroup keeps the centres of one head in LDS, 64 KB of keys' (dim = 128) and
// 64 KB of values', fills a CU with them and looks codes up there: from the L2 each
// centre of 8 bytes would move a line of 128. So the row of all sequences' tiles
// (32 positions) is shared evenly by the workgroups of a head, whatever the
// sequences' lengths are, and a workgroup's share by its waves; what is cut that
// way is joined, in the workgroup at its end and between workgroups by a second
// launch. Workgroup b has head b % heads: with 8 heads each XCD's L2 serves one.
//
// A tile: the centres of its keys are the rows of one matrix operand as they come
// from LDS (v_mfma_f32_16x16x32: a lane holds 8 features of one position), the
// queries the columns of the other; the scores come out with the queries in the
// columns, so that their exponentials are an operand of the product with the
// values without leaving their lanes, the positions being numbered to that end
// (Codes below). The values' rows are features: four features of eight positions,
// looked up, are turned in registers.
//
// 64 sequences of 8192 to 16384 positions, 8 heads of 128 features in sub-vectors of
// 4, 64 query heads: 112 us, 3.5 TB/s of codes (a copy moves 4.8; with the loads of
// codes left out it took 101 of then 111), and the joining launch 5 more. Of a SIMD's
// cycles there vector instructions, 193 a tile and wave with the 16 matrix products
// among them, take 67 %, the products themselves are under way in 21 %; LDS is active
// in 60 % of a CU's (61 % of that bank conflicts, of the random lookups of keys: the
// values' rows are laid out to be free of them). None of them is a limit alone: the
// three waves of a SIMD are issuing for 36 % of their time, ready but not issuing
// for 26 %, and waiting for loads, LDS or a barrier for 39 %. A tile more to every
// wave costs 1.4 us; a launch with one each takes 11 to 13.
#include "kv_device.h"
#include "kv_few.h"

#include <type_traits>

#ifndef KV_SUB
#define KV_SUB 4
#endif
#ifndef KV_FEW
#define KV_FEW 0
#endif

namespace lloyd {

hipError_t launch_kv_few_2(const KvCache &, const KvFew &, const KvFewPlan &, hipStream_t);
hipError_t launch_kv_few_4(const KvCache &, const KvFew &, const KvFewPlan &, hipStream_t);
hipError_t launch_kv_few_8(const KvCache &, const KvFew &, const KvFewPlan &, hipStream_t);
hipError_t launch_kv_attend_2(const KvCache &, const KvAttend &, const KvAttendPlan &, hipStream_t);
hipError_t launch_kv_attend_4(const KvCache &, const KvAttend &, const KvAttendPlan &, hipStream_t);
hipError_t launch_kv_attend_8(const KvCache &, const KvAttend &, const KvAttendPlan &, hipStream_t);

namespace {

// The weights are exp2(score - reference). A new reference lies kLift below the
// largest score, and holds until a score is kLag above that one, when what is
// summed is scaled: weights stay below 2^15, which fp16 holds. For it they are
// lifted, for what is left of small ones is a multiple of 2^-24: a long tail of
// them would lose some of its sum to that.
constexpr float kLag = 8.f;
template <bool FP16>
constexpr float kLift = FP16 ? 7.f : 0.f;

typedef float f4v __attribute__((ext_vector_type(4)));

template <bool FP16>
__device__ inline f4v mfma(u4v a, u4v b, f4v c)
{
    if constexpr (FP16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8v, a),
                                                      __builtin_bit_cast(h8v, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8v, a),
                                                       __builtin_bit_cast(b8v, b), c, 0, 0, 0);
}

// x cut off to fp16, where mask is all ones; 0 where it is 0. (Below the least
// normal number of fp16 the cut leaves more bits than fp16 has there, less than
// 2^-24 that neither part takes up.)
__device__ inline float cut(float x, uint32_t mask)
{
    return __uint_as_float(__float_as_uint(x) & 0xFFFFE000u & mask);
}

// Two numbers cut off to fp16.
__device__ inline uint32_t cut2(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}

// Sizes of one form of the kernel.
template <int D, int SUB>
struct Form {
    static constexpr int S = D / SUB;                  // codes of a head's vector
    static constexpr int SL = S / 4;                   // of them, those of a lane's keys
    static constexpr int VS = SUB < 4 ? SUB : 4;       // features of a value row (granule)
    static constexpr int NG = D / VS;                  // granules
    static constexpr int NH = (NG + 15) / 16;          // rows of 16 granules
    static constexpr int NV = NH * VS;                 // accumulator tiles
    // Waves of the workgroup: as many as the registers allow, 168 each with 12 and
    // 128 with 16 (8 waves: 128 us instead of 111 for the case above; 16 with
    // registers spilled: 138).
    static constexpr int kWaves = kv_waves(D);
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kKeys = D * 512;              // LDS bytes of the key centres: [S][256][SUB]
    static constexpr int kRow = 256;                   // of one code's value centres
    static constexpr int kValues = 256 * kRow;         // of the value centres: [256][D], rows on 256 bytes
    static constexpr int kEntry = NV * 256;            // floats of one wave's accumulators
    // the centres, whose place the waves' last pieces take at the end
    static constexpr int kRoom = kKeys + kValues > kWaves * kEntry * 4 ? kKeys + kValues
                                                                       : kWaves * kEntry * 4;
    static constexpr int kSpans = 1024;                // sequences whose spans are kept in LDS
    // the feature of place x among a wave's accumulators (from D up: none)
    static __device__ int feature(int x)
    {
        const int n = x >> 8, i = (x >> 6) & 3, g = (x >> 4) & 3;
        return (16 * (n / VS) + 4 * g + i) * VS + n % VS;
    }
    static constexpr size_t lds_bytes(int seqs)
    {
        return kRoom + (4 * kWaves * 32 + 3 * kWaves + 2 * kSpans + seqs + 1) * 4;
    }
    static_assert(kRoom + (4 * kWaves * 32 + 3 * kWaves + 2 * kSpans + kKvMaxSeqs + 1) * 4 <= kMaxLds, "LDS");
};

// Positions [start, len) of sequence b, and the 32-position tiles they touch.
struct Span {
    int start, len;
    __device__ int tile0() const { return start >> 5; }
    __device__ int tiles() const { return len > start ? ((len + 31) >> 5) - (start >> 5) : 0; }
};

[[maybe_unused]] __device__ inline Span span_of(const KvCache &c, const KvAttend &a, int b)
{
    const int cap = a.table_pages << c.page_log2;
    Span s;
    s.len = min(max(a.lengths[b], 0), cap);
    s.start = a.starts ? max(a.starts[b], 0) : 0;
    return s;
}

// The workgroups that share a head's tiles: no more than leave each a tile
// for every wave.
__device__ inline int splits_used(int tiles, int splits, int waves)
{
    return min(splits, max(1, (tiles + waves - 1) / waves));
}

// Even shares of n things: where share i of k begins (the first n % k shares
// have one more), and the share that thing t is in.
__device__ inline int share_begin(int n, int i, int k)
{
    return (int)((unsigned)n / (unsigned)k) * i + min(i, (int)((unsigned)n % (unsigned)k));
}

__device__ inline int share_of(int n, int t, int k)
{
    const unsigned each = (unsigned)n / (unsigned)k, more = (unsigned)n % (unsigned)k;
    const unsigned long_end = more * (each + 1);
    return (int)((unsigned)t < long_end ? (unsigned)t / (each + 1) : more + ((unsigned)t - long_end) / each);
}

// Codes of one tile of 32 positions in a lane. Keys: position 8 (r / 4) + 4 t +
// r % 4 (r = lane % 16) for the two products t, codes [SL (lane / 16), + SL).
// Values: granule 16 hh + r, positions [8 (lane / 16), + 8).
template <int D, int SUB>
struct Codes {
    using F = Form<D, SUB>;
    uint32_t k[2][(F::SL + 3) / 4];
    uint32_t v[F::NH][2];
};

template <int N>
__device__ inline void load_bytes(uint32_t *dst, const uint8_t *src)
{
    constexpr int align = N % 16 == 0 ? 16 : N % 8 == 0 ? 8 : N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1;
    dst[(N - 1) / 4] = 0;
    __builtin_memcpy(dst, __builtin_assume_aligned(src, align), N);
}

// base + code n * the size of an entry, in two instructions: base has no bits
// below 256 entries.
template <int SUB>
__device__ inline uint32_t code_offset(const uint32_t *w, int n, uint32_t base)
{
    constexpr int shift = SUB == 2 ? 2 : SUB == 4 ? 3 : 4;
    const int low = 8 * (n & 3);
    const uint32_t at = low < shift ? w[n >> 2] << (shift - low) : w[n >> 2] >> (low - shift);
    return (at & (255u << shift)) | base;
}

// The entry at a byte of LDS (the kernel has no LDS but its dynamic one, which
// so begins at 0), `more` bytes on.
template <int N>
__device__ inline KvEntry<N> lds_entry(uint32_t at, int more = 0)
{
    typedef uint32_t V __attribute__((ext_vector_type(N / 2 > 1 ? N / 2 : 2)));
    typedef std::conditional_t<N == 2, uint32_t, V> T;
    const auto p = (const __attribute__((address_space(3))) char *)(uintptr_t)at;
    return __builtin_bit_cast(KvEntry<N>,
                              *(const __attribute__((address_space(3))) T *)(p + more));
}

// p, worked out here: addresses of what is written once would else be kept in
// registers through the loop before.
template <typename T>
__device__ inline T *here(T *p)
{
    asm volatile("" : "+v"(p));
    return p;
}

// 16 bytes of each lane of a wave from memory to LDS, to the 1024 from `dst` on
// (the same for all lanes), without registers between. A wave's own are there
// after lds_landed(), all waves' after a barrier behind it.
__device__ inline void to_lds16(const void *src, void *dst)
{
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void *)src,
        (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
}

__device__ inline void lds_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The value of the lane N away in its row of 16, around its ends.
template <int N>
__device__ inline float turned(float x)
{
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xF, 0xF, true));
}

// x of rows 0 and 2 of the wave's rows of 16 in both rows of their half, and that
// of rows 1 and 3.
__device__ inline void row_pair(float x, float *even, float *odd)
{
    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *even = __uint_as_float(both[0]);
    *odd = __uint_as_float(both[1]);
}

// Sum of x over the lanes up to this one.
__device__ inline int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);      // 1, 2, 4, 8 lanes down the row
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // rows 0 and 2 to 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);     // the lower half to the upper
    return x;
}

// WIDE: more than 8 queries, so that the high and the low parts of the weights
// are operands of their own. Else the queries stand twice in the 16 columns,
// the first eight of which take the high parts and the others the low ones.
//
// A is KvAttend, or KvFew for few new tokens of every sequence: then what is said of a
// sequence here holds for a unit, up to 8 or 16 (WIDE) query heads of its new tokens,
// each of which sees positions of its own; a row that a unit does not have sees none, so
// that units which are not full (4 query heads of a single token in 8 columns) mask every
// tile, and the scores of one twice. A decode step of 32 sequences of 512 to 4096, 4 heads
// to each of 8 key heads of 128, with distance slopes: 25 us and 4 us for the joining launch; the
// first tile begins 4 to 6 us after the launch does, when the units are known and the centres
// are in LDS.
template <int D, int SUB, bool FP16, bool WIDE, typename A>
__global__ __launch_bounds__((Form<D, SUB>::kThreads)) void
kv_attend_kernel(KvCache c, A a, int splits, int qblocks)
{
    using F = Form<D, SUB>;
    constexpr int W = F::kWaves;
    constexpr bool FEW = std::is_same_v<A, KvFew>;
    constexpr int kUnits = F::kSpans * sizeof(Span) / sizeof(KvUnit);    // kept in LDS
    extern __shared__ uint4 lds[];
    // the values first: their addresses below 2^16 fit the offset of a load
    char *const vbook = reinterpret_cast<char *>(lds);
    char *const kbook = vbook + F::kValues;
    float(*const ml)[32] = reinterpret_cast<float(*)[32]>(vbook + F::kRoom);
    float(*const weight)[32] = ml + 2 * W;
    int *const tag = reinterpret_cast<int *>(ml + 4 * W);
    int *const wave_sum = tag + 2 * W;
    Span *const spans = reinterpret_cast<Span *>(wave_sum + W);          // [kSpans]
    KvUnit *const units = reinterpret_cast<KvUnit *>(spans);             // [kUnits]
    int *const first = reinterpret_cast<int *>(spans + F::kSpans);       // [seqs + 1]

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % c.heads;
    const int qb = blockIdx.x / c.heads % qblocks;
    const int j = blockIdx.x / c.heads / qblocks;
    // of a sequence, of which a unit may have fewer
    const int nq = FEW ? kv_few_rows(WIDE) : min(kKvQueries, a.group - qb * kKvQueries);
    const int rq = WIDE ? r : r & 7;                     // the lane's query
    const int64_t wg = ((int64_t)qb * c.heads + h) * splits + j;
    float *const part_o = a.part_o + wg * (W + 2) * F::kEntry;
    float *const part_ml = a.part_ml + wg * 64;
    constexpr int per16 = 8 / SUB;                       // centres in 16 bytes

    // Where each sequence's tiles begin in the row of all tiles. Up to 64
    // sequences every wave has them in its lanes, and looks nothing up later.
    bool in_lanes = a.seqs <= kWave;
    int tiles, seqs = a.seqs;
    Span my_span{0, 0};
    int my_first = 0, my_next = 0;
    if constexpr (FEW) {
        in_lanes = a.in_lanes;
        if (in_lanes) {
            // the lanes' sequences, then the lanes' units
            KvSeq s{};
            if (lane < a.seqs) s = kv_seq(c, a, lane);
            int b = lane, before = lane;
            if (__any(lane < a.seqs && (unsigned)(s.n * a.group - 1) >= (unsigned)nq)) {
                const int upto = wave_scan((s.n * a.group + nq - 1) / nq);
                seqs = __builtin_amdgcn_readlane(upto, 63);
                if (seqs > kv_most_units(a, nq)) seqs = 0;
                b = 0;
                for (int i = 0; i < a.seqs; ++i) b += __builtin_amdgcn_readlane(upto, i) <= lane;
                before = __shfl(upto, max(b - 1, 0));
                if (b == 0) before = 0;
                s = KvSeq{__shfl(s.t0, b & 63), __shfl(s.n, b & 63), __shfl(s.len, b & 63),
                          __shfl(s.prefix, b & 63)};
            }                                            // else a unit to every sequence
            KvUnit x{};
            if (lane < seqs) x = kv_unit(a, s, b, (lane - before) * nq, nq);
            const int n = x.tiles();
            my_span = Span{x.lo, x.hi};
            my_next = wave_scan(n);
            my_first = my_next - n;
            tiles = __builtin_amdgcn_readlane(my_next, 63);
            if (lane < seqs) {
                first[lane] = my_first;
                units[lane] = x;
                if (blockIdx.x == 0 && wave == 0) a.units.unit[lane] = x;        // for the joining launch
            }
            if (lane == 0) first[seqs] = tiles;
        } else {
            seqs = *a.units.count;
            for (int i = tid; i <= seqs; i += F::kThreads) first[i] = a.units.first[i];
            for (int i = tid; i < min(seqs, kUnits); i += F::kThreads) units[i] = a.units.unit[i];
            tiles = a.units.first[seqs];
            __syncthreads();
        }
    } else if (in_lanes) {
        if (lane < a.seqs) my_span = span_of(c, a, lane);
        const int n = my_span.tiles();
        my_next = wave_scan(n);
        my_first = my_next - n;
        tiles = __builtin_amdgcn_readlane(my_next, 63);
        // all waves write the same, and read it before the others have
        if (lane < a.seqs) {
            first[lane] = my_first;
            spans[lane] = my_span;
        }
        if (lane == 0) first[a.seqs] = tiles;
    } else {
        const int per = (a.seqs + F::kThreads - 1) / F::kThreads;
        int sum = 0;
        for (int i = 0; i < per; ++i) {
            const int b = tid * per + i;
            if (b >= a.seqs) break;
            const Span x = span_of(c, a, b);
            sum += x.tiles();
            if (b < F::kSpans) spans[b] = x;
        }
        const int incl = wave_scan(sum);
        if (lane == 63) wave_sum[wave] = incl;
        __syncthreads();
        const int each = lane < W ? wave_sum[lane] : 0;
        const int upto = wave_scan(each);
        int at = incl - sum + (wave ? __builtin_amdgcn_readlane(upto, wave - 1) : 0);
        tiles = __builtin_amdgcn_readlane(upto, 63);
        for (int i = 0; i < per; ++i) {
            const int b = tid * per + i;
            if (b < a.seqs) {
                first[b] = at;
                at += per == 1 ? sum : span_of(c, a, b).tiles();
            }
        }
        if (tid == 0) first[a.seqs] = tiles;
        __syncthreads();
    }
    const int used = splits_used(tiles, splits, FEW ? kFewShare : W);
    const auto unit_of = [&](int u) {
        if constexpr (FEW) return u < kUnits ? units[u] : a.units.unit[u];
        else return KvUnit{};
    };
    // Where query q of sequence b has its output, and its logarithm among all.
    struct Row {
        int64_t out, lse;
    };
    const auto row_of = [&](int b, int q) {
        if constexpr (FEW) {
            const KvUnit x = unit_of(b);
            const int row = x.row0 + q, token = x.t0 + row / a.group, head = h * a.group + row % a.group;
            return Row{token * a.out_token + head * a.out_head, (int64_t)token * c.heads * a.group + head};
        } else {
            const int head = h * a.group + qb * kKvQueries + q;
            return Row{b * a.out_seq + head * a.out_head, (int64_t)b * c.heads * a.group + head};
        }
    };
    const auto rows_of = [&](int b) {
        if constexpr (FEW) return unit_of(b).rows(a.group, nq);
        else return nq;
    };
    const auto empty = [&](int b) {
        if constexpr (FEW) {
            const int n = rows_of(b);
            for (int i = tid; i < n * D; i += F::kThreads) a.out[row_of(b, i / D).out + i % D] = 0;
            if (a.lse && tid < n) a.lse[row_of(b, tid).lse] = -INFINITY;
        } else {
            for (int i = tid; i < nq * D; i += F::kThreads)
                a.out[b * a.out_seq + (h * a.group + qb * kKvQueries + i / D) * a.out_head + i % D] = 0;
            if (a.lse && tid < nq)
                a.lse[(int64_t)b * c.heads * a.group + h * a.group + qb * kKvQueries + tid] = -INFINITY;
        }
    };
    // Sequences without positions.
    if (in_lanes) {
        uint64_t none = __ballot(lane < seqs && my_first == my_next);
        for (; none; none &= none - 1) {
            const int b = __builtin_ctzll(none);
            if (b % splits == j) empty(b);
        }
    } else {
        for (int b = j; b < seqs; b += splits)
            if (first[b] == first[b + 1]) empty(b);
    }
    if (tid == 0) a.shared[wg] = KvShared{-1, 0};        // unless found below
    if (j >= used) return;
    const int w0 = share_begin(tiles, j, used), w1 = share_begin(tiles, j + 1, used);
    const int a0 = w0 + share_begin(w1 - w0, wave, W), a1 = w0 + share_begin(w1 - w0, wave + 1, W);

    // Final output of query q, feature d of sequence b.
    const auto put = [&](int b, int q, int d, float x) {
        a.out[row_of(b, q).out + d] = (uint16_t)pack2<FP16>(x, 0.f);
    };
    const auto put_lse = [&](int b, int q, float m, float l) {
        if (a.lse)
            a.lse[row_of(b, q).lse] =
                l > 0.f || l != l ? (m + __log2f(l)) * 0.69314718055994531f : -INFINITY;
    };

    f4v acc[F::NV];
    // m: the reference of the exponents (base 2), -inf before the first score
    // above that; m0 is m, or 0 for -inf.
    // l: the lane's part of the sum of the weights.
    float m = -INFINITY, m0 = 0.f, l = 0.f;
    u4v q[D / 32];
    if (lane == 0) { tag[2 * wave] = -1; tag[2 * wave + 1] = -1; }

    // A place in the row of tiles: sequence b, which has tiles [base, next).
    struct Cursor {
        int b, base, next;
        Span sp;
        int of;                  // the sequence that unit b belongs to
    };
    const auto enter = [&](int b) {
        Cursor x;
        x.b = __builtin_amdgcn_readfirstlane(b);
        x.base = __builtin_amdgcn_readfirstlane(first[x.b]);
        x.next = __builtin_amdgcn_readfirstlane(first[x.b + 1]);
        Span s;
        if constexpr (FEW) {
            const KvUnit *const u = x.b < kUnits ? units + x.b : a.units.unit + x.b;
            s = Span{u->lo, u->hi};
            x.of = __builtin_amdgcn_readfirstlane(u->b);
        } else {
            s = x.b < F::kSpans ? spans[x.b] : span_of(c, a, x.b);
        }
        x.sp.start = __builtin_amdgcn_readfirstlane(s.start);
        x.sp.len = __builtin_amdgcn_readfirstlane(s.len);
        return x;
    };
    // to tile t (the next one, below a1)
    const auto advance = [&](Cursor &x, int t) {
        if (t < x.next) return false;
        int b = x.b + 1;
        while (first[b + 1] <= t) ++b;
        x = enter(b);
        return true;
    };
    // Tile t's codes are loaded when those of t - 1 have been looked up, to the
    // same registers, and the numbers of the pages they lie on a tile before.
    struct Where {
        int pos;                 // the tile's first position
        int k_page, v_page;      // numbers of the pages of the lane's keys and values
    };
    // The place of the next numbers to ask for, and of their sequence its row of
    // the table and the first and last entry that may be read (in bytes).
    struct Ahead {
        int pos, low, high;
        const char *row;
    };
    const auto look = [&](const Cursor &x, int t) {
        Ahead y;
        y.pos = (t - x.base + x.sp.tile0()) * 32;
        y.low = x.sp.start >> c.page_log2 << 2;
        y.high = (x.sp.len - 1) >> c.page_log2 << 2;
        y.row = reinterpret_cast<const char *>(a.table + (FEW ? x.of : x.b) * a.table_stride);
        return y;
    };
    const unsigned page_bytes = (unsigned)(c.heads * F::S) << c.page_log2;
    const unsigned last_page = (unsigned)min(c.pages - 1, (int64_t)0x7FFFFFFF);
    // A lane's codes lie at the same place of each of its pages, for tiles begin on
    // multiples of 32 positions; where pages are larger, the tile's place is added.
    const unsigned pm = (1u << c.page_log2) - 1;
    const int64_t head_codes = ((int64_t)h * F::S) << c.page_log2;
    const uint8_t *const k_lane =
        c.k_codes + head_codes + ((8 * (r >> 2) & pm) + (r & 3)) * F::S + g * F::SL;
    const auto v_sub = [&](int hh) {             // of a lane's granule, in its sub-vectors
        return (unsigned)(min(16 * hh + r, F::NG - 1) * F::VS / SUB) << c.page_log2;
    };
    const uint8_t *const v_lane = c.v_codes + head_codes + (8 * g & pm) + v_sub(0);
    const auto v_step = [&](int hh) {            // from granule row 0 to hh: one for all lanes
        return F::NG % 16 == 0 ? (unsigned)(16 * hh * F::VS / SUB) << c.page_log2
                               : v_sub(hh) - v_sub(0);
    };
    const int k_entry = 8 * (r >> 2) >> c.page_log2 << 2, v_entry = 8 * g >> c.page_log2 << 2;
    const auto find = [&](Ahead &y) {
        Where w;
        w.pos = y.pos;
        // groups of 8 positions outside the span: the nearest page inside
        const int at = y.pos >> c.page_log2 << 2;
        w.k_page = *reinterpret_cast<const int32_t *>(
            y.row + (uint32_t)min(max(at + k_entry, y.low), y.high));
        w.v_page = *reinterpret_cast<const int32_t *>(
            y.row + (uint32_t)min(max(at + v_entry, y.low), y.high));
        y.pos += 32;
        return w;
    };
    Codes<D, SUB> cd;            // of the tile at hand, then of the next
    // A number that is no page's is some page's here, never followed out.
    const auto place = [&](const Where &w, int page, int S) {
        return (uint64_t)min((unsigned)page, last_page) * page_bytes + ((unsigned)w.pos & pm) * S;
    };
    const auto load_k = [&](const Where &w) {
        const uint8_t *const k = k_lane + place(w, w.k_page, F::S);
        load_bytes<F::SL>(cd.k[0], k);
        load_bytes<F::SL>(cd.k[1], k + 4 * F::S);
    };
    const auto load_v = [&](const Where &w) {
        const uint8_t *const v = v_lane + place(w, w.v_page, 1);
#pragma unroll
        for (int hh = 0; hh < F::NH; ++hh) load_bytes<8>(cd.v[hh], v + v_step(hh));
    };
    bool changed = false;        // scores are more than products
    if constexpr (FEW) changed = a.cap_log2 > 0.f || a.slopes;
    const float scale = changed ? 1.f : fabsf(a.scale_log2);
    const uint32_t flip = !changed && a.scale_log2 < 0.f ? 0x80008000u : 0u;     // the scale's sign, for the queries
    // what the lane's query of a unit sees, and its slope
    [[maybe_unused]] KvSeen view{0, 0, 0};
    [[maybe_unused]] float slope = 0.f;
    const uint32_t low_parts = r >= 8 ? ~0u : 0u;        // lanes whose columns take them
    // the byte selection that makes the first of two bf16 an fp32 number there, else 0
    const uint32_t low_byte = r >= 8 ? 0x01000C0Cu : 0x0C0C0C0Cu;

    const auto load_q = [&](int b) {
#pragma unroll
        for (int st = 0; st < D / 32; ++st) q[st] = u4v{0, 0, 0, 0};
        if constexpr (FEW) {
            const KvUnit x = unit_of(b);
            view = KvSeen{0, 0, 0};
            slope = 0.f;
            if (rq < x.rows(a.group, nq)) {
                const int t = (x.row0 + rq) / a.group, head = h * a.group + (x.row0 + rq) % a.group;
                const uint16_t *src = a.q + (x.t0 + t) * a.q_token + head * a.q_head + g * (D / 4);
#pragma unroll
                for (int st = 0; st < D / 32; ++st)
                    q[st] = *reinterpret_cast<const u4v *>(src + st * 8);
                view = kv_seen(a, KvSeq{x.t0, x.n, x.len, x.prefix}, t);
                if (a.slopes) slope = a.slopes[head] * kLog2e;
            }
        } else if (rq < nq) {
            const uint16_t *src = a.q + b * a.q_seq +
                                  (h * a.group + qb * kKvQueries + rq) * a.q_head + g * (D / 4);
#pragma unroll
            for (int st = 0; st < D / 32; ++st)
                q[st] = *reinterpret_cast<const u4v *>(src + st * 8);
        }
        m = -INFINITY;
        m0 = 0.f;
        l = 0.f;
#pragma unroll
        for (int n = 0; n < F::NV; ++n) acc[n] = f4v{0.f, 0.f, 0.f, 0.f};
    };
    // Loads come back in order, so the small ones that others hang on go first:
    // page numbers and queries before the centres, the first codes behind them.
    Cursor cur{}, then{};        // of the tile at hand, and of `ahead`
    Ahead ahead{};
    Where where{};
    if (a0 < a1) {
        if (in_lanes) {
            cur.b = (int)__popcll(__ballot(lane < seqs && my_next <= a0));
            cur.base = __builtin_amdgcn_readlane(my_first, cur.b);
            cur.next = __builtin_amdgcn_readlane(my_next, cur.b);
            cur.sp.start = __builtin_amdgcn_readlane(my_span.start, cur.b);
            cur.sp.len = __builtin_amdgcn_readlane(my_span.len, cur.b);
            if constexpr (FEW) cur.of = __builtin_amdgcn_readfirstlane(units[cur.b].b);
        } else {
            // the last b with first[b] <= a0: of every 64th, then of the 64
            const int block = __popcll(__ballot(first[min((lane + 1) * kWave, seqs)] <= a0));
            const int b = min(block * kWave + lane + 1, seqs);
            cur = enter(block * kWave + __popcll(__ballot(first[b] <= a0)));
        }
        then = cur;
        ahead = look(then, a0);
        where = find(ahead);
        load_q(cur.b);
    }
    // The centres of this head, entries from K up zeros. With all 256 the keys'
    // are one run of bytes and go straight to LDS, 16 to a lane; the values'
    // go through registers, to be turned to one row of all features for each
    // code.
    constexpr int rounds = (D * 32 + F::kThreads - 1) / F::kThreads;
    static_assert(D * 32 % kWave == 0, "whole waves");
    const uint16_t *const ks = c.k_centres + (int64_t)h * F::S * c.K * SUB;
    const uint16_t *const vs = c.v_centres + (int64_t)h * F::S * c.K * SUB;
    // lanes: 4 runs of 16 bytes in each of 16 sub-vectors, for whole sectors
    // from memory and few conflicts in LDS
    const auto value_s = [&](int i) { return ((i * F::kThreads + tid) >> 2) % F::S; };
    const auto value_code = [&](int i) {
        const int n = i * F::kThreads + tid;
        return ((n >> 2) / F::S * 4 + (n & 3)) * per16;
    };
    u4v vreg[rounds];                                    // (as uint4, they went to memory)
    if (c.K == 256) {
#pragma unroll
        for (int i = 0; i < rounds; ++i) {
            const int at = (i * F::kThreads + (wave << 6)) * 16;         // of the wave's first lane
            if (at < F::kKeys) to_lds16(reinterpret_cast<const char *>(ks) + at + lane * 16, kbook + at);
        }
#pragma unroll
        for (int i = 0; i < rounds; ++i)
            if (i * F::kThreads + tid < D * 32)
                vreg[i] = *reinterpret_cast<const u4v *>(vs + (value_s(i) * 256 + value_code(i)) * SUB);
    } else {
        using E = KvEntry<SUB>;
#pragma unroll 4
        for (int i = tid; i < F::S * 256; i += F::kThreads) {
            const int s = i >> 8, code = i & 255;
            E ke{}, ve{};
            if (code < c.K) {
                ke = kv_load<SUB>(ks + (s * c.K + code) * SUB);
                ve = kv_load<SUB>(vs + (s * c.K + code) * SUB);
            }
            reinterpret_cast<E *>(kbook)[i] = ke;
            *reinterpret_cast<E *>(vbook + code * F::kRow + s * (SUB * 2)) = ve;
        }
    }
    if (a0 < a1) {
        load_k(where);
        load_v(where);
        if (a0 + 1 < a1) {
            if (advance(then, a0 + 1)) ahead = look(then, a0 + 1);
            where = find(ahead);
        }
    }
    if (c.K == 256) {
#pragma unroll
        for (int i = 0; i < rounds; ++i) {
            if (i * F::kThreads + tid >= D * 32) break;
#pragma unroll
            for (int x = 0; x < per16; ++x) {
                KvEntry<SUB> e;
#pragma unroll
                for (int y = 0; y < SUB / 2; ++y) e.w[y] = vreg[i][x * (SUB / 2) + y];
                *reinterpret_cast<KvEntry<SUB> *>(vbook + (value_code(i) + x) * F::kRow +
                                                  value_s(i) * (SUB * 2)) = e;
            }
        }
    }
    lds_landed();
    __syncthreads();

    if (a0 < a1) {
        const uint32_t k_base = F::kValues + g * (F::SL * 512 * SUB);
        // One tile of 32 positions from `pos` on. What the span leaves out of it
        // is masked in branches of its own, which most tiles skip (of single tokens'
        // attention and of full units).
        const auto step = [&](int t, int pos) {
            const Span &sp = cur.sp;
            bool partial = pos < sp.start || pos + 32 > sp.len;
            if constexpr (FEW) partial = !__all(pos >= view.lo && pos + 32 <= view.hi);
            const auto seen = [&](int i) {
                const int p = pos + 8 * g + i;
                return p >= sp.start && p < sp.len;
            };
            const auto sees = [&](int i) {               // the lane's query
                const int p = pos + 8 * g + i;
                if constexpr (FEW) return p >= view.lo && p < view.hi;
                else return seen(i);
            };
            // All centres of the tile are asked for before any is waited for: a
            // lookup takes far longer than its turn, and a SIMD has but three waves
            // (four with dim = 64).
            KvEntry<SUB> ke[2][F::SL];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < F::SL; ++n)
                    ke[u][n] = lds_entry<SUB>(code_offset<SUB>(cd.k[u], n, k_base), n * (512 * SUB));
            __builtin_amdgcn_sched_barrier(0);
            const Where coming = where;
            if (t + 1 < a1) load_k(coming);
            if (t + 2 < a1) {
                if (advance(then, t + 2)) ahead = look(then, t + 2);
                where = find(ahead);
            }
            // scores: rows are positions, columns queries
            float z[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                f4v s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int st = 0; st < D / 32; ++st) {
                    u4v op;
#pragma unroll
                    for (int i = 0; i < 4; ++i) op[i] = ke[u][(st * 8 + 2 * i) / SUB].w[i % (SUB / 2)];
                    s = mfma<FP16>(op, q[st], s);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * u + i] = s[i];
            }
            __builtin_amdgcn_sched_barrier(0);
            KvEntry<F::VS> ve[F::NH][8];
#pragma unroll
            for (int hh = 0; hh < F::NH; ++hh)
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    // code * 256 + the granule's place in the row, in one byte selection
                    ve[hh][x] = lds_entry<F::VS>(
                        __builtin_amdgcn_perm(cd.v[hh][x >> 2],
                                              (uint32_t)(min(16 * hh + r, F::NG - 1) * F::VS * 2),
                                              0x0C0C0000u | (4 + (x & 3)) << 8));
            __builtin_amdgcn_sched_barrier(0);
            if (t + 1 < a1) load_v(coming);
            if constexpr (FEW) {
                if (a.cap_log2 > 0.f) {
                    kv_cap<8>(z, a);
                } else if (changed) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] *= a.scale_log2;
                }
                if (a.slopes) {
                    const float far = (float)(view.at - pos - 8 * g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = __builtin_fmaf(-slope, fabsf(far - (float)i), z[i]);
                }
            }
            if (partial) {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = sees(i) ? z[i] : -INFINITY;
            }
            float top = fmaxf(z[0], z[1]);
#pragma unroll
            for (int i = 2; i < 8; ++i) top = fmaxf(top, z[i]);
            top *= scale;
            if (__any(!(top <= m + (kLag + kLift<FP16>)))) {      // NaN included
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                top = fmaxf(top - kLift<FP16>, m);
                m0 = top == -INFINITY ? 0.f : top;
                const float alpha = __builtin_amdgcn_exp2f(m - m0);
                m = top;
                l *= alpha;
#pragma unroll
                for (int n = 0; n < F::NV; ++n) acc[n] *= alpha;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = __builtin_fmaf(z[i], scale, -m0);
            if (partial) {                                // again: a scale of 0 gave NaN
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = sees(i) ? z[i] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                z[i] = __builtin_amdgcn_exp2f(z[i]);
                l += z[i];
            }
            // Each weight as the sum of two 16-bit numbers. One alone (8 bits of bf16)
            // would cost as much of the result as its own final rounding. Of bf16 both
            // are rounded to nearest: cut off, 16 bits would leave every weight too
            // small, 8e-6 of it on average, beside a sum l that has all of it (three
            // parts, 24 bits, change the outputs no further and take 8 % longer). Of
            // fp16 they are cut, which leaves 2^-21 at most.
            u4v p, p_lo;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float z0 = z[2 * i], z1 = z[2 * i + 1];
                if constexpr (FP16 && WIDE) {
                    p[i] = cut2(z0, z1);
                    p_lo[i] = cut2(z0 - cut(z0, ~0u), z1 - cut(z1, ~0u));
                } else if constexpr (FP16) {
                    p[i] = cut2(z0 - cut(z0, low_parts), z1 - cut(z1, low_parts));
                } else if constexpr (WIDE) {
                    p[i] = pack2<FP16>(z0, z1);
                    p_lo[i] = pack2<FP16>(z0 - __uint_as_float(p[i] << 16),
                                          z1 - __uint_as_float(p[i] & 0xFFFF0000u));
                } else {
                    const uint32_t high = pack2<FP16>(z0, z1);
                    p[i] = pack2<FP16>(
                        z0 - __uint_as_float(__builtin_amdgcn_perm(0u, high, low_byte)),
                        z1 - __uint_as_float(high & low_parts & 0xFFFF0000u));
                }
            }
            // values: rows are features, columns queries
#pragma unroll
            for (int hh = 0; hh < F::NH; ++hh) {
                KvEntry<F::VS> (&e)[8] = ve[hh];
                if (partial) {                            // 0 weighs nothing, not 0 * NaN
#pragma unroll
                    for (int x = 0; x < 8; ++x)
#pragma unroll
                        for (int w = 0; w < F::VS / 2; ++w) e[x].w[w] = seen(x) ? e[x].w[w] : 0u;
                }
#pragma unroll
                for (int i = 0; i < F::VS; ++i) {
                    u4v op;
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        op[x] = __builtin_amdgcn_perm(e[2 * x + 1].w[i / 2], e[2 * x].w[i / 2],
                                                      i % 2 ? 0x07060302u : 0x05040100u);
                    f4v &o = acc[hh * F::VS + i];
                    if (WIDE) o = mfma<FP16>(op, p_lo, o);
                    o = mfma<FP16>(op, p, o);
                }
            }
        };

        // A sequence's tiles of the wave at a time, the work on a tile in a loop of
        // its own, which so keeps its registers.
        int turn = (wave >> 2) % 3;
        for (int t = a0; t < a1;) {
            const int b = cur.b, piece = t, end = min(cur.next, a1);
#pragma unroll
            for (int st = 0; st < D / 32; ++st) q[st] ^= flip;
            int pos = (t - cur.base + cur.sp.tile0()) * 32;
            for (; t < end; ++t) {
                // The SIMD's waves take turns at the highest priority: the oldest
                // would have it always, end first and leave the last ones to
                // run alone. There are three turns; of four waves (dim = 64) two
                // share one.
                if (turn == 0) __builtin_amdgcn_s_setprio(2);
                else if (turn == 1) __builtin_amdgcn_s_setprio(1);
                else __builtin_amdgcn_s_setprio(0);
                turn = turn == 2 ? 0 : turn + 1;
                step(t, pos);
                pos += 32;
            }
            float lw = l + __shfl_xor(l, 16);
            lw += __shfl_xor(lw, 32);
            if (!WIDE) {
#pragma unroll
                for (int n = 0; n < F::NV; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[n][i] += turned<8>(acc[n][i]);
            }
            if (piece == cur.base && end == cur.next) {  // the whole sequence
                const float inv = lw > 0.f || lw != lw ? 1.f / lw : 0.f;
                if (r < rows_of(b)) {
                    uint16_t *const dst = here(a.out + row_of(b, r).out + 4 * g * F::VS);
#pragma unroll
                    for (int n = 0; n < F::NV; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int d = (16 * (n / F::VS) + i) * F::VS + n % F::VS;
                            if (d + 4 * g * F::VS < D)
                                dst[d] = (uint16_t)pack2<FP16>(acc[n][i] * inv, 0.f);
                        }
                    if (g == 0) put_lse(b, r, m, lw);
                }
            } else {
                const int e = 2 * wave + (end == a1);
                if (lane == 0) tag[e] = b;
                if (g == 0) { ml[e][r] = m; ml[e][16 + r] = lw; }
                if (end != a1) {
                    float *const dst = here(part_o + wave * F::kEntry + lane);
#pragma unroll
                    for (int n = 0; n < F::NV; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[(n * 4 + i) * 64] = acc[n][i];
                }
            }
            if (end < a1) {
                advance(cur, end);
                load_q(cur.b);
            }
        }
    }
    __syncthreads();
    // The centres are done with: their place takes each wave's last piece.
    float *const last = reinterpret_cast<float *>(lds);
    if (tag[2 * wave + 1] >= 0) {
#pragma unroll
        for (int n = 0; n < F::NV; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                last[wave * F::kEntry + (n * 4 + i) * 64 + lane] = acc[n][i];
    }
    __syncthreads();
    // Piece e = 2 * wave is the one before a wave's last, e + 1 its last. Those of
    // one sequence are last pieces of waves that follow each other, and at most
    // one that the next wave ended. All of this runs once a launch, when its
    // instructions come from memory: it is kept short.
    static_assert(W >= 8 && W <= 16, "two queries to each of 8 waves, pieces to half a wave");
    if (wave < 8) {
        // lanes: pieces; halves: queries. The pieces' weights against the
        // sequence's largest reference, and the sequence's sum.
        const int e = lane & 31, qq = 2 * wave + (lane >> 5);
        const int b = e < 2 * W ? tag[e] : -1;
        const float em = e < 2 * W ? ml[e][qq] : 0.f, el = e < 2 * W ? ml[e][16 + qq] : 0.f;
        const int at = b >= 0 ? first[b] : 0, end = b >= 0 ? first[b + 1] : 0;
        for (uint64_t todo = __ballot(b >= 0); todo;) {
            const int lead = __builtin_ctzll(todo);
            const bool in = b == __builtin_amdgcn_readlane(b, lead);
            todo &= ~__ballot(in);
            float top = in ? em : -INFINITY;
            top = fmaxf(top, turned<1>(top));
            top = fmaxf(top, turned<2>(top));
            top = fmaxf(top, turned<4>(top));
            top = fmaxf(top, turned<8>(top));
            float even, odd;
            row_pair(top, &even, &odd);
            top = fmaxf(even, odd);
            const float w = __builtin_amdgcn_exp2f(em - (top == -INFINITY ? 0.f : top));
            float lw = in ? el * w : 0.f;
            lw += turned<1>(lw);
            lw += turned<2>(lw);
            lw += turned<4>(lw);
            lw += turned<8>(lw);
            row_pair(lw, &even, &odd);
            lw = even + odd;
            if (!in) continue;
            weight[e][qq] = w;
            weight[e][16 + qq] = lw;
            if (e != lead || qq >= rows_of(b)) continue;
            if (at >= w0 && end <= w1) {
                put_lse(b, qq, top, lw);
            } else {
                const int slot = at < w0 ? 0 : 1;
                part_ml[slot * 32 + qq] = top;
                part_ml[slot * 32 + 16 + qq] = lw;
            }
        }
    }
    __syncthreads();
    constexpr int mine = (F::kEntry + F::kThreads - 1) / F::kThreads;
    const int qq = tid & 15;
    const int tag_of = lane < 2 * W ? tag[lane] : -1;
    const int at_of = tag_of >= 0 ? first[tag_of] : 0, end_of = tag_of >= 0 ? first[tag_of + 1] : 0;
    uint64_t todo = __ballot(tag_of >= 0);
#pragma unroll 1
    while (todo) {
        const int lead = __builtin_ctzll(todo), b = __builtin_amdgcn_readlane(tag_of, lead);
        const int at_b = __builtin_amdgcn_readlane(at_of, lead);
        const int end_b = __builtin_amdgcn_readlane(end_of, lead);
        const uint64_t in = __ballot(tag_of == b);
        todo &= ~in;
        float o[mine] = {}, lw = 0.f;
        if (const uint64_t heads = in & 0x5555555555555555ull) {
            const int e = __builtin_ctzll(heads);
            const float w = weight[e][qq];
            lw = weight[e][16 + qq];
#pragma unroll
            for (int i = 0; i < mine; ++i)
                o[i] = w * part_o[(e >> 1) * F::kEntry + min(i * F::kThreads + tid, F::kEntry - 1)];
        }
        if (const uint64_t lasts = in & 0xAAAAAAAAAAAAAAAAull) {
            const int from = __builtin_ctzll(lasts) >> 1, to = (63 - __builtin_clzll(lasts)) >> 1;
            lw = weight[2 * from + 1][16 + qq];
#pragma unroll 1
            for (int n = from; n <= to; n += 4) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int at = min(n + k, to);       // the last again, with no weight
                    const float w = n + k <= to ? weight[2 * at + 1][qq] : 0.f;
#pragma unroll
                    for (int i = 0; i < mine; ++i)
                        o[i] += w * last[at * F::kEntry + min(i * F::kThreads + tid, F::kEntry - 1)];
                }
            }
        }
        const bool whole = at_b >= w0 && end_b <= w1;
        const int slot = at_b < w0 ? 0 : 1;
        const float inv = lw > 0.f || lw != lw ? 1.f / lw : 0.f;
#pragma unroll
        for (int i = 0; i < mine; ++i) {
            const int at = i * F::kThreads + tid, d = F::feature(at);
            if (qq < rows_of(b) && at < F::kEntry) {
                if (!whole)
                    part_o[(W + slot) * F::kEntry + at] = o[i];
                else if (d < D)
                    put(b, qq, d, o[i] * inv);
            }
        }
        if (!whole && slot && tid == 0)
            a.shared[wg] = KvShared{b, share_of(tiles, end_b - 1, used) - j + 1};
    }
}

// Joins what the workgroups left of the sequences that several shared. Joining
// workgroup j of a head takes the sequence that begins in share j and does not
// end there, if there is one: its parts are that share's second and the first
// of the shares after it. It takes 256 of the outputs, one to a thread, and asks
// for the parts and for what weighs them at once: this launch is a chain of two
// trips to memory.
template <int D, int SUB, bool FP16, typename A>
__global__ __launch_bounds__(256) void kv_join_kernel(KvCache c, A a, int splits)
{
    using F = Form<D, SUB>;
    constexpr bool FEW = std::is_same_v<A, KvFew>;
    constexpr int chunks = F::kEntry / 256, batch = 8;
    const int x = blockIdx.x % chunks * 256 + threadIdx.x;
    const int j = blockIdx.x / chunks % (splits - 1), hq = blockIdx.x / chunks / (splits - 1);
    const int h = hq % c.heads, qb = hq / c.heads;
    int nq = FEW ? 0 : min(kKvQueries, a.group - qb * kKvQueries);
    const int64_t wg = (int64_t)hq * splits + j;
    const int tid = threadIdx.x, q = tid & 15;
    const auto part = [&](int i) {                       // of this thread's output
        return a.part_o[((wg + i) * (F::kWaves + 2) + F::kWaves + (i == 0)) * F::kEntry + x];
    };
    const auto ml = [&](int i) { return a.part_ml + (wg + i) * 64 + (i == 0) * 32 + q; };
    // Most such sequences have two parts: those are asked for along with what says
    // so (there is a share after this one).
    const int i0 = tid >> 4;
    float in[batch];
    in[0] = part(0);
    in[1] = part(1);
    float m0 = *ml(min(i0, 1)), l0 = ml(min(i0, 1))[16];
    const KvShared found = a.shared[wg];
    if (found.b < 0) return;
    const int b = found.b, n = found.parts;              // 2 <= n <= splits <= kCUs
    if (n > 2) {
#pragma unroll
        for (int k = 2; k < batch; ++k) in[k] = part(min(k, n - 1));
        if (i0 >= 2 && i0 < n) {
            m0 = *ml(i0);
            l0 = ml(i0)[16];
        }
    } else {
#pragma unroll
        for (int k = 2; k < batch; ++k) in[k] = 0.f;
    }
    // weight of each part, for each query: [part][query]
    __shared__ float weight[kCUs * 16];
    __shared__ float s_top[16 * 16], s_sum[16 * 16];
    float top = i0 < n ? m0 : -INFINITY;
    for (int i = i0 + 16; i < n; i += 16) {
        const float v = *ml(i);
        weight[i * 16 + q] = v;
        top = fmaxf(top, v);
    }
    s_top[tid] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s_top[i * 16 + q]);
    const float safe = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    if (i0 < n) {
        const float w = __builtin_amdgcn_exp2f(m0 - safe);
        sum = w * l0;
        weight[i0 * 16 + q] = w;
    }
    for (int i = i0 + 16; i < n; i += 16) {
        const float w = __builtin_amdgcn_exp2f(weight[i * 16 + q] - safe);
        sum += w * ml(i)[16];
        weight[i * 16 + q] = w;
    }
    s_sum[tid] = sum;
    __syncthreads();
    float lw = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) lw += s_sum[i * 16 + q];
    int token = b, head = h * a.group + qb * kKvQueries + q;
    if constexpr (FEW) {
        const KvUnit u = a.units.unit[b];
        nq = u.rows(a.group, a.rows);
        token = u.t0 + (u.row0 + q) / a.group;
        head = h * a.group + (u.row0 + q) % a.group;
    }
    if (q >= nq) return;
    if (x < 16 && a.lse)
        a.lse[(int64_t)token * c.heads * a.group + head] =
            lw > 0.f || lw != lw ? (top + __log2f(lw)) * 0.69314718055994531f : -INFINITY;
    const int d = F::feature(x);
    if (d >= D) return;
    float o = 0.f;
#pragma unroll 1
    for (int i = 0; i < n; i += batch) {
        float now[batch];
#pragma unroll
        for (int k = 0; k < batch; ++k) now[k] = in[k];
        if (i + batch < n)
#pragma unroll
            for (int k = 0; k < batch; ++k) in[k] = part(min(i + batch + k, n - 1));
#pragma unroll
        for (int k = 0; k < batch; ++k)
            if (i + k < n) o += weight[(i + k) * 16 + q] * now[k];
    }
    int64_t stride;
    if constexpr (FEW) stride = a.out_token;
    else stride = a.out_seq;
    a.out[token * stride + head * a.out_head + d] =
        (uint16_t)pack2<FP16>(lw > 0.f || lw != lw ? o / lw : 0.f, 0.f);
}

template <int D, int SUB, bool FP16, bool WIDE, typename A>
hipError_t launch(const KvCache &c, const A &a, int splits, int qblocks, int seqs, hipStream_t s)
{
    using F = Form<D, SUB>;
    const unsigned grid = (unsigned)c.heads * qblocks * splits;
    hipLaunchKernelGGL((kv_attend_kernel<D, SUB, FP16, WIDE, A>), dim3(grid), dim3(F::kThreads),
                       F::lds_bytes(seqs), s, c, a, splits, qblocks);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    hipLaunchKernelGGL((kv_join_kernel<D, SUB, FP16, A>),
                       dim3((unsigned)c.heads * qblocks * (splits - 1) * (F::kEntry / 256)), dim3(256), 0,
                       s, c, a, splits);
    return hipGetLastError();
}

template <int D, bool WIDE, typename A>
hipError_t launch_type(const KvCache &c, const A &a, int splits, int qblocks, int seqs, hipStream_t s)
{
    return c.fp16 ? launch<D, KV_SUB, true, WIDE>(c, a, splits, qblocks, seqs, s)
                  : launch<D, KV_SUB, false, WIDE>(c, a, splits, qblocks, seqs, s);
}

template <bool WIDE, typename A>
hipError_t launch_dim(const KvCache &c, const A &a, int splits, int qblocks, int seqs, hipStream_t s)
{
    return c.dim == 64 ? launch_type<64, WIDE>(c, a, splits, qblocks, seqs, s)
         : c.dim == 96 ? launch_type<96, WIDE>(c, a, splits, qblocks, seqs, s)
                       : launch_type<128, WIDE>(c, a, splits, qblocks, seqs, s);
}

#if KV_SUB == 2
// Workgroups of a head and block of queries: one to a CU, for the centres fill its LDS,
// and no more than leave each wave a tile.
int splits_of(const KvCache &c, int qblocks, int64_t tiles)
{
    int64_t splits = (int64_t)kCUs / (c.heads * qblocks);
    const int waves = kv_waves(c.dim);
    if (splits > (tiles + waves - 1) / waves) splits = (tiles + waves - 1) / waves;
    return splits < 1 ? 1 : (int)splits;
}

// Floats of a wave's accumulators.
size_t entry_of(const KvCache &c)
{
    const int gran = c.sub < 4 ? c.sub : 4;
    return (size_t)((c.dim / gran + 15) / 16 * gran) * 256;
}
#endif

}  // namespace

#define KV_CAT2(a, b) a##b
#define KV_CAT(a, b) KV_CAT2(a, b)
#if KV_FEW
hipError_t KV_CAT(launch_kv_few_, KV_SUB)(const KvCache &c, const KvFew &a, const KvFewPlan &p,
                                          hipStream_t s)
{
    return p.wide ? launch_dim<true>(c, a, p.splits, 1, p.units, s)
                  : launch_dim<false>(c, a, p.splits, 1, p.units, s);
}
#else
hipError_t KV_CAT(launch_kv_attend_, KV_SUB)(const KvCache &c, const KvAttend &a,
                                             const KvAttendPlan &p, hipStream_t s)
{
    return a.group > kKvQueries / 2 ? launch_dim<true>(c, a, p.splits, p.qblocks, a.seqs, s)
                                    : launch_dim<false>(c, a, p.splits, p.qblocks, a.seqs, s);
}
#endif

#if KV_SUB == 2 && !KV_FEW
KvAttendPlan plan_kv_attend(const KvCache &c, int seqs, int group, int64_t table_pages)
{
    KvAttendPlan p{};
    p.qblocks = (group + kKvQueries - 1) / kKvQueries;
    const int64_t span = table_pages << c.page_log2;
    p.splits = splits_of(c, p.qblocks, seqs * ((span + kKvTile - 1) / kKvTile));
    const size_t entry = entry_of(c) * sizeof(float);
    const size_t wgs = (size_t)c.heads * p.qblocks * p.splits;
    const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    p.shared_off = 0;
    p.part_o_off = up(wgs * sizeof(KvShared));
    p.part_ml_off = p.part_o_off + wgs * (kv_waves(c.dim) + 2) * entry;
    p.total = p.part_ml_off + up(wgs * 64 * sizeof(float));
    return p;
}

hipError_t launch_kv_attend(const KvCache &c, const KvAttend &a, const KvAttendPlan &p,
                            hipStream_t s)
{
    return c.sub == 2 ? launch_kv_attend_2(c, a, p, s)
         : c.sub == 4 ? launch_kv_attend_4(c, a, p, s) : launch_kv_attend_8(c, a, p, s);
}
#endif

#if KV_SUB == 2 && KV_FEW
KvFewPlan plan_kv_few(const KvCache &c, const KvNew &n)
{
    KvFewPlan p{};
    const int64_t rows = n.tokens * n.group;
    // what fits half the columns takes half the products (and twice the queries' registers):
    // in us, by half and whole columns, 37 and 44 (64 sequences of 2000, 8 rows), 38 and 39 (32
    // of 4096, 4 rows), 30 and 38 (32 of 4096, 8 rows)
    p.wide = rows > 8 * (int64_t)n.seqs;
    const int64_t units = kv_most_units(n, kv_few_rows(p.wide));
    p.units = units > kKvMaxFew ? kKvMaxFew + 1 : (int)units;
    p.in_lanes = n.seqs <= kWave && units <= kWave;
    const int64_t span = ((int64_t)n.table_pages << c.page_log2) / kKvTile + 1;
    p.splits = splits_of(c, 1, units * span);
    if (p.splits > 1) {
        const int64_t most = kCUs / c.heads, tiles = units * span;
        p.splits = (int)(most < 1 ? 1 : most * kFewShare < tiles ? most : (tiles + kFewShare - 1) / kFewShare);
    }
    const size_t wgs = (size_t)c.heads * p.splits;
    p.total = 0;
    for (size_t x : {sizeof(int32_t), sizeof(int32_t) * (p.units + 1), sizeof(KvUnit) * p.units,
                     sizeof(KvShared) * wgs, wgs * 64 * sizeof(float),
                     wgs * (kv_waves(c.dim) + 2) * entry_of(c) * sizeof(float)})
        p.total += (x + 255) / 256 * 256;
    return p;
}

hipError_t launch_kv_few(const KvCache &c, const KvNew &n, const KvTokensOut &o, const KvFewPlan &p,
                         void *ws, hipStream_t s)
{
    char *at = static_cast<char *>(ws);
    const auto take = [&](size_t bytes) {
        char *const x = at;
        at += (bytes + 255) / 256 * 256;
        return x;
    };
    const size_t wgs = (size_t)c.heads * p.splits;
    KvFew a{};
    static_cast<KvNew &>(a) = n;
    a.out = o.out;
    a.out_token = o.out_token;
    a.out_head = o.out_head;
    a.lse = o.lse;
    a.in_lanes = p.in_lanes;
    a.rows = kv_few_rows(p.wide);
    a.units.count = reinterpret_cast<int32_t *>(take(sizeof(int32_t)));
    a.units.first = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * (p.units + 1)));
    a.units.unit = reinterpret_cast<KvUnit *>(take(sizeof(KvUnit) * p.units));
    a.shared = reinterpret_cast<KvShared *>(take(sizeof(KvShared) * wgs));
    a.part_ml = reinterpret_cast<float *>(take(wgs * 64 * sizeof(float)));
    a.part_o = reinterpret_cast<float *>(take(0));
    if (!p.in_lanes) {
        const hipError_t e = launch_kv_units(c, n, a.units, kv_few_rows(p.wide), s);
        if (e != hipSuccess) return e;
    }
    return c.sub == 2 ? launch_kv_few_2(c, a, p, s)
         : c.sub == 4 ? launch_kv_few_4(c, a, p, s) : launch_kv_few_8(c, a, p, s);
}
#endif

}  // namespace lloyd
