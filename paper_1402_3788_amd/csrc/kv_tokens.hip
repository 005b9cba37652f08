// Attention of many new tokens of every sequence over the cache of codes.
//
// One query to a wave: 64 positions at a time, one to a lane for the scores, the
// features over the lanes for the sum of the values.
#include "kv_tokens_device.h"

namespace lloyd {

namespace {

template <int SUB, bool FP16>
__global__ __launch_bounds__(kWave) void kv_tokens_kernel(KvCache c, KvNew a, KvTokensOut o)
{
    __shared__ uint16_t q[128];
    __shared__ float weight[kWave];
    __shared__ int pages[kWave];
    const int lane = threadIdx.x, heads = c.heads * a.group, S = c.dim / SUB;
    const int hq = blockIdx.x % heads, t = blockIdx.x / heads, h = hq / a.group;
    int b = 0;
    KvSeq s{};
    for (; b < a.seqs; ++b) {
        s = kv_seq(c, a, b);
        if (t >= s.t0 && t < s.t0 + s.n) break;
    }
    if (b == a.seqs) return;
    for (int i = lane; i < c.dim; i += kWave) q[i] = a.q[t * a.q_token + hq * a.q_head + i];
    __syncthreads();
    const KvSeen x = kv_seen(a, s, t - s.t0);
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    const int last = (int)min(c.pages - 1, (int64_t)0x7FFFFFFF), mask = (1 << c.page_log2) - 1;
    for (int at = x.lo; at < x.hi; at += kWave) {
        const int pos = at + lane;
        float z = -INFINITY;
        int page = 0;
        if (pos < x.hi) {
            page = min((uint32_t)a.table[b * a.table_stride + (pos >> c.page_log2)], (uint32_t)last);
            const uint8_t *codes = c.k_codes + kv_head(c, page, h, S) + (int64_t)(pos & mask) * S;
            float dot = 0.f;
            for (int n = 0; n < S; ++n) {
                const int code = codes[n];
                if (code >= c.K) continue;
                float k[SUB];
                kv_unpack<FP16>(kv_load<SUB>(c.k_centres + ((int64_t)(h * S + n) * c.K + code) * SUB), k);
                for (int e = 0; e < SUB; ++e) dot = __builtin_fmaf(k[e], kv_float<FP16>(q[n * SUB + e]), dot);
            }
            z = a.cap_log2 > 0.f ? kv_capped(dot * a.scale_cap, a.cap_log2) : dot * a.scale_log2;
            if (a.slopes) z -= a.slopes[hq] * kLog2e * (float)abs(x.at - pos);
        }
        float top = z;
        for (int k = 1; k < kWave; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
        top = fmaxf(top, m);
        const float m0 = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(m - m0);
        m = top;
        const float p = pos < x.hi ? __builtin_amdgcn_exp2f(z - m0) : 0.f;
        float sum = p;
        for (int k = 1; k < kWave; k *= 2) sum += __shfl_xor(sum, k);
        l = l * alpha + sum;
        acc[0] *= alpha;
        acc[1] *= alpha;
        weight[lane] = p;
        pages[lane] = page;
        __syncthreads();
        for (int i = 0; i < min(kWave, x.hi - at); ++i) {
            const float p1 = weight[i];
            const uint8_t *codes = c.v_codes + kv_head(c, pages[i], h, S) + ((at + i) & mask);
            for (int e = 0; e < 2; ++e) {
                const int d = lane + 64 * e;
                if (d >= c.dim) break;
                const int code = codes[(d / SUB) << c.page_log2];
                if (code < c.K)
                    acc[e] += p1 * kv_float<FP16>(c.v_centres[((int64_t)(h * S + d / SUB) * c.K + code) * SUB + d % SUB]);
            }
        }
        __syncthreads();
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    for (int e = 0; e < 2; ++e) {
        const int d = lane + 64 * e;
        if (d >= c.dim) break;
        uint16_t r;
        if constexpr (FP16) r = __builtin_bit_cast(uint16_t, (_Float16)(acc[e] * inv));
        else r = __builtin_bit_cast(uint16_t, (__bf16)(acc[e] * inv));
        o.out[t * o.out_token + hq * o.out_head + d] = r;
    }
    if (o.lse && lane == 0)
        o.lse[(int64_t)t * heads + hq] = l > 0.f || l != l ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

template <int SUB>
hipError_t launch(const KvCache &c, const KvNew &n, const KvTokensOut &o, hipStream_t s)
{
    const auto kernel = c.fp16 ? kv_tokens_kernel<SUB, true> : kv_tokens_kernel<SUB, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(n.tokens * c.heads * n.group)), dim3(kWave), 0, s, c, n, o);
    return hipGetLastError();
}

}  // namespace

size_t kv_attend_tokens_bytes(const KvCache &, const KvNew &) { return 256; }

hipError_t launch_kv_attend_tokens(const KvCache &c, const KvNew &n, const KvTokensOut &o, void *,
                                   hipStream_t s)
{
    return c.sub == 2 ? launch<2>(c, n, o, s) : c.sub == 4 ? launch<4>(c, n, o, s) : launch<8>(c, n, o, s);
}

}  // namespace lloyd
