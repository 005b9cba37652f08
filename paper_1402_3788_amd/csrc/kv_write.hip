// Encoding of keys and values into the cache: every sub-vector x gets the number
// of its nearest centre (Eq. (2), in the fp32 operations kmeans.h states).
//
// The matrix cores screen: score_j = x . c_j - |c_j|^2 / 2, the largest of which
// belongs to the nearest centre but for rounding. What rounding can do is bounded:
//   products of 16-bit numbers are exact in fp32; up to 11 of them and of the
//   parts of |c|^2 / 2 are added, each addition off by at most 2^-23 of the
//   magnitudes summed (no more than faithful rounding assumed), and |c|^2 / 2 by
//   10 such units of itself, so a score is off by E <= 21 * 2^-23 (|x|^2 + |c|^2);
//   the stated distance is off by 6.5 * 2^-24 of itself, itself <= 2 (|x|^2 + |c|^2).
// So the centre that the definition chooses scores at least the best score less
// 2 E + 6.5 * 2^-23 (|x|^2 + C^2) < 2^-17 (|x|^2 + C^2), C the largest |c|. The
// groups of 16 centres whose best score is not below that are evaluated as the
// definition says, nearly always one group of the 16. Where a bound is not a
// number (overflow, NaN) every group is.
//
// A sub-vector costs 128 scores to a lane at half an instruction each (the
// maximum of three), and 8 distances at 18: the vector ALU bounds it. 4096 tokens
// of 8 heads of 128 features in sub-vectors of 4 (2.1 million of 256 centres):
// FIGURE.
#include "kv_device.h"

namespace lloyd {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kSubs = 4;             // sub-vectors of a workgroup: a dword of key codes
constexpr int kTokens = 32;          // tokens of a wave's step, columns of the product

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef _Float16 h4v __attribute__((ext_vector_type(4)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));

// What a lane holds of a matrix operand: 8 values for SUB = 8, else 4. A centre
// is padded to it with zeros; so is the record of -|c|^2 / 2 as three bf16
// numbers that add up to it.
template <int SUB>
struct alignas(SUB == 8 ? 16 : 8) Operand {
    uint32_t w[SUB == 8 ? 4 : 2];
};

template <int SUB>
__device__ inline f16v product(bool fp16, const Operand<SUB> &a, const Operand<SUB> &b, f16v c)
{
    if constexpr (SUB == 8)
        return fp16 ? __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8v, a),
                                                             __builtin_bit_cast(h8v, b), c, 0, 0, 0)
                    : __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8v, a),
                                                              __builtin_bit_cast(b8v, b), c, 0, 0, 0);
    else
        return fp16 ? __builtin_amdgcn_mfma_f32_32x32x8f16(__builtin_bit_cast(h4v, a),
                                                           __builtin_bit_cast(h4v, b), c, 0, 0, 0)
                    : __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(__builtin_bit_cast(s4v, a),
                                                               __builtin_bit_cast(s4v, b), c, 0, 0, 0);
}

__device__ inline uint32_t bf16_bits(float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x); }

// A workgroup takes kSubs sub-vectors of one head of the keys or the values
// (their centres in LDS), and of the tokens the steps y, y + gridDim.y, ...
template <int SUB, bool FP16>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache c, KvTokens t)
{
    __shared__ Operand<SUB> centre[kSubs][256];
    __shared__ Operand<SUB> half_norm[kSubs][256];
    __shared__ float largest[kSubs][kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int S = c.dim / SUB, groups = S / kSubs;
    const int s0 = (int)(blockIdx.x % groups) * kSubs;
    const int h = (int)(blockIdx.x / groups) % c.heads;
    const bool values = (int)(blockIdx.x / groups) >= c.heads;
    const uint16_t *const centres = (values ? c.v_centres : c.k_centres) +
                                    ((int64_t)h * S + s0) * c.K * SUB;
#pragma unroll 1
    for (int s = 0; s < kSubs; ++s) {
        // one centre to a thread
        static_assert(kThreads == 256, "");
        Operand<SUB> op{}, rec{};
        float norm = 0.f;
        if (tid < c.K) {
            const KvEntry<SUB> e = kv_load<SUB>(centres + (s * c.K + tid) * SUB);
            float y[SUB];
            kv_unpack<FP16>(e, y);
#pragma unroll
            for (int i = 0; i < SUB / 2; ++i) op.w[i] = e.w[i];
#pragma unroll
            for (int i = 0; i < SUB; ++i) norm = __builtin_fmaf(y[i], y[i], norm);
            const float n = -0.5f * norm;
            const uint32_t hi = bf16_bits(n);
            const float n1 = n - __uint_as_float(hi << 16);
            const uint32_t mid = bf16_bits(n1);
            const float n2 = n1 - __uint_as_float(mid << 16);
            rec.w[0] = hi | mid << 16;
            rec.w[1] = bf16_bits(n2);
            if (!(norm < INFINITY)) rec.w[0] = rec.w[1] = 0;     // every group is evaluated
        } else {
            rec.w[0] = 0xFF7Fu;                                  // no centre: never the best
        }
        centre[s][tid] = op;
        half_norm[s][tid] = rec;
        for (int d = 32; d; d /= 2) norm = fmaxf(norm, __shfl_xor(norm, d));
        if (lane == 0) largest[s][wave] = norm;
    }
    __syncthreads();

    const int col = lane & 31, up = lane >> 5;
    const int tiles = (c.K + 31) >> 5;
    const int64_t stride = (int64_t)gridDim.y * (kWaves * kTokens);
    for (int64_t first = (int64_t)blockIdx.y * (kWaves * kTokens) + wave * kTokens; first < t.tokens;
         first += stride) {
        const int64_t tok = first + col;
        int64_t page = 0;
        int off = 0;
        const bool live = tok < t.tokens && kv_slot(c, t.slots[tok], &page, &off);
        const int64_t from = live ? tok : first;
        const uint16_t *const src = (values ? t.v + from * t.v_token + h * t.v_head
                                            : t.k + from * t.k_token + h * t.k_head) + s0 * SUB;
        KvEntry<SUB> in[kSubs];
        __builtin_memcpy(in, __builtin_assume_aligned(src, 16), sizeof(in));
        uint32_t codes = 0;
#pragma unroll 1
        for (int s = 0; s < kSubs; ++s) {
            float x[SUB];
            KvEntry<SUB> e = in[0];
#pragma unroll
            for (int i = 1; i < kSubs; ++i)
                if (s == i) e = in[i];
            kv_unpack<FP16>(e, x);
            float norm = 0.f;
#pragma unroll
            for (int i = 0; i < SUB; ++i) norm = __builtin_fmaf(x[i], x[i], norm);
            // columns of the product: tokens. bf16: the lower lanes' values are x,
            // the upper ones' take the three parts of the norm; fp16: a product for each.
            Operand<SUB> bx{}, ones{};
            if (FP16 || up == 0)
#pragma unroll
                for (int i = 0; i < SUB / 2; ++i) bx.w[i] = FP16 && up ? 0u : e.w[i];
            if (FP16 ? up == 0 : up == 1) {
                ones.w[0] = 0x3F803F80u;
                ones.w[1] = 0x3F80u;
            }
            if (!FP16 && up) bx = ones;
            const Operand<SUB> *const a = !FP16 && up ? half_norm[s] : centre[s];
            float top[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                top[n] = -INFINITY;
                if (n >= tiles) continue;
                f16v d = {};
                if (FP16) {
                    Operand<4> rec, one;
                    rec.w[0] = half_norm[s][n * 32 + col].w[0];
                    rec.w[1] = half_norm[s][n * 32 + col].w[1];
                    one.w[0] = ones.w[0];
                    one.w[1] = ones.w[1];
                    d = product<4>(false, rec, one, d);
                }
                d = product<SUB>(FP16, a[n * 32 + col], bx, d);
                float m = fmaxf(d[0], d[1]);
#pragma unroll
                for (int i = 2; i < 16; ++i) m = fmaxf(m, d[i]);
                top[n] = m;
            }
            float best = top[0];
#pragma unroll
            for (int n = 1; n < 8; ++n) best = fmaxf(best, top[n]);
            best = fmaxf(best, __shfl_xor(best, 32));
            const float big = fmaxf(fmaxf(largest[s][0], largest[s][1]),
                                    fmaxf(largest[s][2], largest[s][3]));
            const float least = best - (0x1p-17f * (norm + big) + 1e-30f);
            // bit n: rows 32 n + 8 i + 0..3 for i = 0..3; bit 8 + n: those + 4
            uint32_t open = 0;
#pragma unroll
            for (int n = 0; n < 8; ++n)
                if (n < tiles && !(top[n] < least)) open |= 1u << n;
            const uint32_t other = __shfl_xor(open, 32);
            open = up ? open << 8 | other : open | other << 8;
            // both lanes of a token evaluate half of a group's 16 centres each
            float near = INFINITY;
            int code = 0;
            while (__any(open)) {
                if (open) {
                    const int bit = __builtin_ctz(open);
                    open &= open - 1;
                    const int row = (bit & 7) * 32 + (bit >> 3) * 4 + up * 16;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int j = row + (k >> 2) * 8 + (k & 3);
                        KvEntry<SUB> ce;
                        const Operand<SUB> o = centre[s][j];
#pragma unroll
                        for (int i = 0; i < SUB / 2; ++i) ce.w[i] = o.w[i];
                        float y[SUB];
                        kv_unpack<FP16>(ce, y);
                        const float d = kv_distance(x, y);
                        if (j < c.K && (d < near || (d == near && j < code))) {
                            near = d;
                            code = j;
                        }
                    }
                }
            }
            const float near2 = __shfl_xor(near, 32);
            const int code2 = __shfl_xor(code, 32);
            if (near2 < near || (near2 == near && code2 < code)) code = code2;
            codes |= (uint32_t)code << (8 * s);
        }
        if (!live) continue;
        const int64_t head = (page * c.heads + h) << c.page_log2;
        if (!values) {
            if (!up)
                *reinterpret_cast<uint32_t *>(c.k_codes + (head + off) * S + s0) = codes;
        } else {
            uint8_t *const dst = c.v_codes + head * S + off;
#pragma unroll
            for (int s = 0; s < 2; ++s)
                dst[(int64_t)(s0 + 2 * up + s) << c.page_log2] = (uint8_t)(codes >> (8 * (2 * up + s)));
        }
    }
}

template <int SUB>
hipError_t launch(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    const unsigned kinds = 2 * c.heads * (c.dim / SUB / kSubs);
    const int64_t steps = (t.tokens + kWaves * kTokens - 1) / (kWaves * kTokens);
    // enough workgroups for every CU to hold several, no more: each loads centres
    const int64_t most = (8 * kCUs + kinds - 1) / kinds;
    const unsigned y = (unsigned)(steps < most ? steps : most);
    if (c.fp16)
        hipLaunchKernelGGL((kv_write_kernel<SUB, true>), dim3(kinds, y), dim3(kThreads), 0, s, c, t);
    else
        hipLaunchKernelGGL((kv_write_kernel<SUB, false>), dim3(kinds, y), dim3(kThreads), 0, s, c, t);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    return c.sub == 2 ? launch<2>(c, t, s) : c.sub == 4 ? launch<4>(c, t, s) : launch<8>(c, t, s);
}

}  // namespace lloyd
