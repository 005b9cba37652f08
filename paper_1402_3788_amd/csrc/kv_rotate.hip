// Rotary positions of queries and keys.
//
// A pair of features (a, b) turns by w = position * frequency: two products and two
// sums to 8 bytes that move, so the bytes bound it. A workgroup takes a token: its
// angles are reduced to part of a turn in fp64 (at position 2^20 an fp32 angle is off
// by 0.03), their cosines and sines go to LDS once for all heads, and each thread
// turns 16 features, 8 of each kind, of one head after the other.
#include "kv_device.h"
#include "kv_tokens.h"

namespace lloyd {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 256;

typedef uint32_t u4v __attribute__((ext_vector_type(4)));

template <bool FP16>
__device__ inline uint32_t round16(float x)
{
    if constexpr (FP16)
        return __builtin_bit_cast(uint16_t, (_Float16)x);
    else
        return __builtin_bit_cast(uint16_t, (__bf16)x);
}

template <bool FP16>
__device__ inline float low16(uint32_t w) { return kv_float<FP16>(w & 0xFFFFu); }
template <bool FP16>
__device__ inline float high16(uint32_t w) { return kv_float<FP16>(w >> 16); }

// (cos, sin) of the angle of pair i, times the amplitude.
__device__ inline float2 turn_of(const KvRotate &r, int64_t position, int i)
{
    // in turns; the product is rounded to 2^-53 of itself, as the angle is
    const double w = (double)position * r.frequencies[i] * 0.15915494309189533577;
    const float x = 2.f * (float)(w - rint(w));
    float s, c;
    sincospif(x, &s, &c);
    return make_float2(r.amplitude * c, r.amplitude * (r.inverse ? -s : s));
}

// Features in runs of 8 where pairs fall on whole runs of 16 bytes; else one pair
// after the other.
template <bool FP16, bool INTERLEAVED, bool RUNS>
__global__ __launch_bounds__(kThreads) void kv_rotate_kernel(KvRotate r, int parts)
{
    __shared__ float2 turns[kMaxHalf];
    const int tid = threadIdx.x, part = blockIdx.x % parts;
    const int heads = r.x[0].heads + r.x[1].heads;
    const int64_t step = gridDim.x / parts;
    for (int64_t t = blockIdx.x / parts; t < r.tokens; t += step) {
        if (r.half) {
            const int64_t at = r.positions[t];
            __syncthreads();                                 // the last token's are done with
            for (int i = tid; i < r.half; i += kThreads) turns[i] = turn_of(r, at, i);
            __syncthreads();
        }
        const auto head_of = [&](int h, const uint16_t **from, uint16_t **to) {
            const KvTurned &x = h < r.x[0].heads ? r.x[0] : r.x[1];
            const int64_t hh = h < r.x[0].heads ? h : h - r.x[0].heads;
            *from = x.from + t * x.from_token + hh * x.from_head;
            *to = x.to + t * x.to_token + hh * x.to_head;
        };
        if constexpr (RUNS) {
            // a run of each half, or two runs side by side; then runs that are copied
            const int turned = r.half / 8, units = turned + (r.dim / 8 - 2 * turned);
            for (int u = part * kThreads + tid; u < heads * units; u += parts * kThreads) {
                const int h = u / units, i = u - h * units;
                const uint16_t *from;
                uint16_t *to;
                head_of(h, &from, &to);
                if (i >= turned) {
                    const int at = 8 * (i + turned);
                    *reinterpret_cast<u4v *>(to + at) = *reinterpret_cast<const u4v *>(from + at);
                    continue;
                }
                const int at0 = INTERLEAVED ? 16 * i : 8 * i, at1 = INTERLEAVED ? at0 + 8 : at0 + r.half;
                u4v x = *reinterpret_cast<const u4v *>(from + at0);
                u4v y = *reinterpret_cast<const u4v *>(from + at1);
                if constexpr (INTERLEAVED) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 c0 = turns[8 * i + k], c1 = turns[8 * i + 4 + k];
                        const float a0 = low16<FP16>(x[k]), b0 = high16<FP16>(x[k]);
                        const float a1 = low16<FP16>(y[k]), b1 = high16<FP16>(y[k]);
                        x[k] = round16<FP16>(a0 * c0.x - b0 * c0.y) | round16<FP16>(a0 * c0.y + b0 * c0.x) << 16;
                        y[k] = round16<FP16>(a1 * c1.x - b1 * c1.y) | round16<FP16>(a1 * c1.y + b1 * c1.x) << 16;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 c0 = turns[8 * i + 2 * k], c1 = turns[8 * i + 2 * k + 1];
                        const float a0 = low16<FP16>(x[k]), a1 = high16<FP16>(x[k]);
                        const float b0 = low16<FP16>(y[k]), b1 = high16<FP16>(y[k]);
                        x[k] = round16<FP16>(a0 * c0.x - b0 * c0.y) | round16<FP16>(a1 * c1.x - b1 * c1.y) << 16;
                        y[k] = round16<FP16>(a0 * c0.y + b0 * c0.x) | round16<FP16>(a1 * c1.y + b1 * c1.x) << 16;
                    }
                }
                *reinterpret_cast<u4v *>(to + at0) = x;
                *reinterpret_cast<u4v *>(to + at1) = y;
            }
        } else {
            const int units = r.half + (r.dim - 2 * r.half);
            for (int u = part * kThreads + tid; u < heads * units; u += parts * kThreads) {
                const int h = u / units, i = u - h * units;
                const uint16_t *from;
                uint16_t *to;
                head_of(h, &from, &to);
                if (i >= r.half) {
                    to[i + r.half] = from[i + r.half];
                    continue;
                }
                const int at0 = INTERLEAVED ? 2 * i : i, at1 = INTERLEAVED ? at0 + 1 : at0 + r.half;
                const float a = kv_float<FP16>(from[at0]), b = kv_float<FP16>(from[at1]);
                const float2 c = turns[i];
                to[at0] = (uint16_t)round16<FP16>(a * c.x - b * c.y);
                to[at1] = (uint16_t)round16<FP16>(a * c.y + b * c.x);
            }
        }
    }
}

template <bool FP16>
hipError_t launch(const KvRotate &r, hipStream_t s)
{
    const int heads = r.x[0].heads + r.x[1].heads;
    // few tokens: a token's heads over several workgroups, that repeat its angles
    int parts = 1;
    while (r.tokens * parts < 2 * kCUs && heads * (r.dim / 16) > parts * kThreads) ++parts;
    const bool runs = r.half % 8 == 0;
    const auto kernel = r.interleaved
                            ? (runs ? kv_rotate_kernel<FP16, true, true> : kv_rotate_kernel<FP16, true, false>)
                            : (runs ? kv_rotate_kernel<FP16, false, true> : kv_rotate_kernel<FP16, false, false>);
    const int64_t most = (int64_t)1 << 20;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((r.tokens < most ? r.tokens : most) * parts)),
                       dim3(kThreads), 0, s, r, parts);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_rotate(const KvRotate &r, hipStream_t s)
{
    return r.fp16 ? launch<true>(r, s) : launch<false>(r, s);
}

}  // namespace lloyd
