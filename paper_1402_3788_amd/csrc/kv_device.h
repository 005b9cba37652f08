// Device helpers of the key-value cache kernels.
#pragma once

#include "kv.h"

namespace lloyd {

// One 16-bit value as fp32 (exact).
template <bool FP16>
__device__ inline float kv_float(uint32_t bits)
{
    if constexpr (FP16)
        return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    else
        return __uint_as_float(bits << 16);
}

// SUB packed 16-bit features, two to a dword.
template <int SUB>
struct alignas(SUB * 2) KvEntry {
    uint32_t w[SUB / 2];
};

template <int SUB>
__device__ inline KvEntry<SUB> kv_load(const uint16_t *p)
{
    KvEntry<SUB> e;
    __builtin_memcpy(&e, __builtin_assume_aligned(p, SUB * 2), SUB * 2);
    return e;
}

template <bool FP16, int SUB>
__device__ inline void kv_unpack(const KvEntry<SUB> &e, float (&v)[SUB])
{
#pragma unroll
    for (int i = 0; i < SUB; ++i) v[i] = kv_float<FP16>((e.w[i / 2] >> (16 * (i & 1))) & 0xFFFFu);
}

// Eq. (2) in the order include/kmeans.h states: every operation rounded,
// neighbours added first.
template <int SUB>
__device__ inline float kv_distance(const float (&x)[SUB], const float (&c)[SUB])
{
    float d[SUB];
#pragma unroll
    for (int i = 0; i < SUB; ++i) {
        const float e = x[i] - c[i];
        d[i] = e * e;
    }
#pragma unroll
    for (int n = SUB / 2; n >= 1; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) d[i] = d[2 * i] + d[2 * i + 1];
    return d[0];
}

// What lanes of a wave wrote to LDS before it, other lanes read after it. A wave's
// LDS instructions are carried out in order: it keeps the compiler's order only.
__device__ inline void kv_wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A slot's page and the token's place in it; false for a slot that is not in the
// cache.
__device__ inline bool kv_slot(const KvCache &c, int64_t slot, uint32_t *page, uint32_t *off)
{
    *page = (uint32_t)(slot >> c.page_log2);
    *off = (uint32_t)slot & ((1u << c.page_log2) - 1);
    return (uint64_t)slot < (uint64_t)c.pages << c.page_log2;
}

// Codes before those of head h on a page; S of them to a token.
__device__ inline int64_t kv_head(const KvCache &c, uint32_t page, int h, int S)
{
    return (uint64_t)page * ((uint32_t)(c.heads * S) << c.page_log2) +
           ((uint32_t)(h * S) << c.page_log2);
}

}  // namespace lloyd
