// Rotary positions of queries and keys.
//
// A pair of features (a, b) turns by w = position * frequency: two products and two
// sums to 8 bytes that move, so the bytes bound it. A workgroup takes a token: its
// angles are reduced to part of a turn in fp64 (at position 2^20 an fp32 angle is off
// by 0.03), their cosines and sines go to LDS once for all heads, and each thread turns
// runs of 8 features, 16 bytes, of one head after the other. Pairs side by side lie in a
// run. Pairs half of the turned part apart lie in two runs that one thread has where that
// half is whole runs; otherwise the partners come over LDS. 8192 tokens of 72 heads of
// 128 features, bf16: 58 us, 5.2 TB/s of reads and writes, a copy's rate. 40 heads, whose 168 MB
// the last-level cache holds from one pass to the next: 27 us, 6.2 TB/s, side by side or half
// of it apart; 36 us with 46 features turned over LDS, where one pair at a time to a thread,
// with its loads and stores of 2 bytes, took 111.
#include "kv_device.h"
#include "kv_tokens.h"

namespace lloyd {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 256;
constexpr int kWaves = kThreads / kWave;
// what a wave has in LDS: 64 runs of 8, with room for words that lie over their ends
constexpr int kWaveRow = 8 + 64 * 8 + 16;

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

// Where a pair's features lie: side by side, half of the turned part apart and that whole
// runs of 16 bytes, or any other half apart.
enum { kInterleaved, kRuns, kOdd };

template <bool FP16, int FORM>
__global__ __launch_bounds__(kThreads) void kv_rotate_kernel(KvRotate r, int parts)
{
    __shared__ float2 turns[kMaxHalf];
    __shared__ __attribute__((aligned(16))) uint16_t wave_rows[FORM == kOdd ? kWaves * kWaveRow : 1];
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
        if constexpr (FORM == kInterleaved) {
            const int units = r.dim / 8;
            for (int u = part * kThreads + tid; u < heads * units; u += parts * kThreads) {
                const int h = u / units, i = u - h * units;
                const uint16_t *from;
                uint16_t *to;
                head_of(h, &from, &to);
                u4v x = *reinterpret_cast<const u4v *>(from + 8 * i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 c = turns[4 * i + k < r.half ? 4 * i + k : 0];
                    const float a = low16<FP16>(x[k]), b = high16<FP16>(x[k]);
                    const uint32_t y = round16<FP16>(a * c.x - b * c.y) | round16<FP16>(a * c.y + b * c.x) << 16;
                    x[k] = 4 * i + k < r.half ? y : x[k];
                }
                *reinterpret_cast<u4v *>(to + 8 * i) = x;
            }
        } else if constexpr (FORM == kRuns) {
            // a run of each half, then runs that are copied
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
                const int at0 = 8 * i, at1 = at0 + r.half;
                u4v x = *reinterpret_cast<const u4v *>(from + at0);
                u4v y = *reinterpret_cast<const u4v *>(from + at1);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 c0 = turns[8 * i + 2 * k], c1 = turns[8 * i + 2 * k + 1];
                    const float a0 = low16<FP16>(x[k]), a1 = high16<FP16>(x[k]);
                    const float b0 = low16<FP16>(y[k]), b1 = high16<FP16>(y[k]);
                    x[k] = round16<FP16>(a0 * c0.x - b0 * c0.y) | round16<FP16>(a1 * c1.x - b1 * c1.y) << 16;
                    y[k] = round16<FP16>(a0 * c0.y + b0 * c0.x) | round16<FP16>(a1 * c1.y + b1 * c1.x) << 16;
                }
                *reinterpret_cast<u4v *>(to + at0) = x;
                *reinterpret_cast<u4v *>(to + at1) = y;
            }
        } else {
            // a thread's 8 features stay its own; their partners, half of the turned part
            // away, come over LDS in whole words, an odd way off shifted by half of one
            const int lane = tid % kWave, wave = tid / kWave, units = r.dim / 8, rows = kWave / units;
            const int row = lane / units, i = lane - row * units;
            uint16_t *const mine = wave_rows + wave * kWaveRow + 8 + 8 * lane;
            const auto away = [&](int by, uint32_t (&w)[4]) {
                const uint32_t *const p = reinterpret_cast<const uint32_t *>(mine + (by - (by & 1)));
                uint32_t v[5];
#pragma unroll
                for (int k = 0; k < 5; ++k) v[k] = p[k];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = by & 1 ? __builtin_amdgcn_alignbit(v[k + 1], v[k], 16) : v[k];
            };
            for (int h0 = (part * kWaves + wave) * rows; h0 < heads; h0 += parts * kWaves * rows) {
                const bool there = row < rows && h0 + row < heads;
                const uint16_t *from;
                uint16_t *to;
                head_of(there ? h0 + row : h0, &from, &to);
                u4v x{};
                if (there) {
                    x = *reinterpret_cast<const u4v *>(from + 8 * i);
                    *reinterpret_cast<u4v *>(mine) = x;
                }
                asm volatile("" ::: "memory");           // a wave's LDS accesses keep their order
                __builtin_amdgcn_wave_barrier();
                uint32_t up[4] = {}, down[4] = {};
                if (there && 8 * i < r.half) away(r.half, up);
                if (there && 8 * i + 7 >= r.half && 8 * i < 2 * r.half) away(-r.half, down);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int at = 8 * i + k;
                    const bool first = at < r.half;
                    const float2 c = turns[min(first ? at : at - r.half, r.half - 1)];
                    const uint32_t other = first ? up[k / 2] : down[k / 2];
                    const float a = k % 2 ? high16<FP16>(x[k / 2]) : low16<FP16>(x[k / 2]);
                    const float b = k % 2 ? high16<FP16>(other) : low16<FP16>(other);
                    const uint32_t y = round16<FP16>(a * c.x + b * (first ? -c.y : c.y));
                    const uint32_t both = k % 2 ? (x[k / 2] & 0xFFFFu) | y << 16 : (x[k / 2] & 0xFFFF0000u) | y;
                    x[k / 2] = at < 2 * r.half ? both : x[k / 2];
                }
                asm volatile("" ::: "memory");
                __builtin_amdgcn_wave_barrier();
                if (there) *reinterpret_cast<u4v *>(to + 8 * i) = x;
            }
        }
    }
}

template <bool FP16>
hipError_t launch(const KvRotate &r, hipStream_t s)
{
    const int heads = r.x[0].heads + r.x[1].heads;
    // few tokens: a token's heads over several workgroups, that repeat its angles (one token of
    // 72 heads of 128 2.6 us, in one workgroup 4.0; of 256 heads 2.6 and 7.8)
    int parts = 1;
    while (r.tokens * parts < 2 * kCUs && heads * (r.dim / 16) > parts * kThreads) ++parts;
    const auto kernel = r.interleaved ? kv_rotate_kernel<FP16, kInterleaved>
                      : r.half % 8 == 0 ? kv_rotate_kernel<FP16, kRuns> : kv_rotate_kernel<FP16, kOdd>;
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
