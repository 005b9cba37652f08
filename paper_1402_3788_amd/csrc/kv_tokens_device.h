// Device helpers of the kernels that take many new tokens (kv_tokens.hip, kv_weigh.hip).
#pragma once

#include "kv_device.h"
#include "kv_tokens.h"

namespace lloyd {

typedef float f2v __attribute__((ext_vector_type(2)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef __bf16 b2v __attribute__((ext_vector_type(2)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));

// 32 rows by 32 columns by 16: a lane holds k = 8 (lane / 32) to + 7 of row, or column,
// lane % 32; of the product, rows 8 (i / 4) + 4 (lane / 32) + i % 4 of column lane % 32.
template <bool FP16>
__device__ inline f16v mfma32(u4v a, u4v b, f16v c)
{
    if constexpr (FP16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8v, a),
                                                      __builtin_bit_cast(h8v, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8v, a),
                                                       __builtin_bit_cast(b8v, b), c, 0, 0, 0);
}

template <bool FP16>
__device__ inline uint32_t pack2(float a, float b)
{
    const f2v v = {a, b};
    if constexpr (FP16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2v));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2v));
}

// 4, 8 or 16 bytes at a byte of LDS, `more` bytes on.
template <int N>
struct LdsWords {
    typedef uint32_t type __attribute__((ext_vector_type(N / 4)));
};
template <>
struct LdsWords<4> {
    typedef uint32_t type;
};

template <typename T>
__device__ inline T lds_get(uint32_t at, int more = 0)
{
    typedef const __attribute__((address_space(3))) typename LdsWords<sizeof(T)>::type *P;
    return __builtin_bit_cast(T, *(P)((const __attribute__((address_space(3))) char *)(uintptr_t)at + more));
}

template <typename T>
__device__ inline void lds_put(uint32_t at, int more, const T &x)
{
    typedef typename LdsWords<sizeof(T)>::type W;
    typedef __attribute__((address_space(3))) W *P;
    *(P)((__attribute__((address_space(3))) char *)(uintptr_t)at + more) = __builtin_bit_cast(W, x);
}

// All waves' LDS accesses before it are done behind it; loads and stores of memory stay
// under way, which __syncthreads() would wait for.
__device__ inline void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The larger, or the sum, of a lane's and that of the lane 32 away.
__device__ inline float max_halves(float x)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

__device__ inline float sum_halves(float x)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(both[0]) + __uint_as_float(both[1]);
}

// Sum of x over the lanes up to this one.
__device__ inline int scan_lanes(int x)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 1; k < kWave; k *= 2) {
        const int y = __shfl_up(x, k);
        if (lane >= k) x += y;
    }
    return x;
}

// The new tokens [t0, t0 + n) of a sequence and its cached positions.
struct KvSeq {
    int t0, n, len, prefix;
};

__device__ inline KvSeq kv_seq(const KvCache &c, const KvNew &a, int b)
{
    const int T = (int)a.tokens, cap = a.table_pages << c.page_log2;
    KvSeq s;
    s.t0 = min(max(a.bounds[b], 0), T);
    s.n = min(max(a.bounds[b + 1], s.t0), T) - s.t0;
    s.len = min(max(a.lengths[b], 0), cap);
    s.prefix = a.prefixes ? min(a.prefixes[b], s.len) : 0;
    return s;
}

// Positions [lo, hi) that token i of a sequence (number t0 + i) sees; lo < hi or
// both 0. Its own is at.
struct KvSeen {
    int lo, hi, at;
};

// (of token i, whose start is given)
__device__ inline KvSeen kv_seen(const KvNew &a, const KvSeq &s, int i, int start)
{
    KvSeen x;
    x.at = s.len - s.n + i;
    x.hi = max(x.at + 1, s.prefix);
    x.lo = max(start, 0);
    if (a.window) x.lo = max(x.lo, x.at - a.window + 1);
    if (x.lo >= x.hi) x.lo = x.hi = 0;
    return x;
}

__device__ inline KvSeen kv_seen(const KvNew &a, const KvSeq &s, int i)
{
    return kv_seen(a, s, i, a.starts ? a.starts[s.t0 + i] : 0);
}

// cap * tanh(scale * z / cap) to base 2, of a lane's N products z. With x = scale * z / cap,
// up to 5/8 tanh x = x + x^3 P(x^2), P of degree 4 fitted to it there (off by 2^-27 of it);
// beyond 1 - 2 / (1 + e^2x), which for small x would be off by 2^-23 of 1, 4e-6 of a score for
// a cap of 50. The two ranges and their forms are Moshier's (Methods and Programs for
// Mathematical Functions, 1989), the coefficients a fit of this file's own. Most scores are far below their cap: a wave whose scores all are saves the
// exponentials.
template <int N, typename V>
__device__ inline void kv_cap(V &z, const KvNew &a)
{
    float x[N], most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = z[i] * a.scale_cap;
        most = fmaxf(most, fabsf(x[i]));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = x[i] * x[i], y = a.cap_log2 * x[i];
        float p = __builtin_fmaf(t, -0.0057036951f, 0.020637562f);
        p = __builtin_fmaf(t, p, -0.053739071f);
        p = __builtin_fmaf(t, p, 0.13331431f);
        p = __builtin_fmaf(t, p, -0.33333281f);
        z[i] = __builtin_fmaf(y * t, p, y);
    }
    if (__any(!(most <= 0.625f))) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float e = __builtin_amdgcn_exp2f(x[i] * (2.f * kLog2e));
            const float far = a.cap_log2 - 2.f * a.cap_log2 * __builtin_amdgcn_rcpf(1.f + e);
            z[i] = fabsf(x[i]) <= 0.625f ? z[i] : far;
        }
    }
}

// Rows [row0, row0 + up to as many as a unit has) of sequence b, whose new tokens are
// [t0, t0 + n): the positions that any of them sees lie in [lo, hi).
struct KvUnit {
    int b, row0, t0, n, len, prefix, lo, hi;
    __device__ int tile0() const { return lo >> 5; }
    __device__ int tiles() const { return hi > lo ? ((hi + 31) >> 5) - (lo >> 5) : 0; }
    __device__ int rows(int group, int most) const { return min(n * group - row0, most); }
};

// The unit of up to `rows` rows of sequence b from row0 on.
__device__ inline KvUnit kv_unit(const KvNew &a, const KvSeq &s, int b, int row0, int rows)
{
    const int i0 = row0 / a.group, i1 = (min(row0 + rows, s.n * a.group) - 1) / a.group;
    int lo = INT32_MAX, hi = 0;
    if (a.starts) {
        for (int i = i0; i <= i1; ++i) {
            const KvSeen y = kv_seen(a, s, i);
            if (y.hi > 0) lo = min(lo, y.lo);
            hi = max(hi, y.hi);
        }
    } else {
        // bounds rise from token to token
        hi = kv_seen(a, s, i1).hi;
        for (int i = i0; i <= i1 && lo == INT32_MAX; ++i) {
            const KvSeen y = kv_seen(a, s, i);
            if (y.hi > 0) lo = y.lo;
        }
    }
    return KvUnit{b, row0, s.t0, s.n, s.len, s.prefix, lo < hi ? lo : 0, lo < hi ? hi : 0};
}

// Units and where each one's tiles begin among all (one more than there are units).
struct KvUnits {
    int32_t *count;
    int32_t *first;
    KvUnit *unit;
};

}  // namespace lloyd
