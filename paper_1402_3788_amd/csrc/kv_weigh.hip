// The weight that attention gave to cached positions.
//
// One position of one head to a thread, whose key is looked up once.
#include "kv_tokens_device.h"

namespace lloyd {

namespace {

constexpr int kThreads = 256;

template <int SUB, bool FP16>
__global__ __launch_bounds__(kThreads) void kv_weigh_kernel(KvCache c, KvNew a, KvWeigh w, int chunks)
{
    const int b = blockIdx.x / chunks / c.heads, h = blockIdx.x / chunks % c.heads;
    const int64_t pos64 = (int64_t)(blockIdx.x % chunks) * kThreads + threadIdx.x;
    if (pos64 >= w.positions) return;
    const int pos = (int)pos64, S = c.dim / SUB;
    float *const to = w.weights + b * w.weights_seq + h * w.weights_head + pos;
    const KvSeq s = kv_seq(c, a, b);
    float sum = 0.f;
    if (pos < s.len) {
        const int page = min((uint32_t)a.table[b * a.table_stride + (pos >> c.page_log2)], (uint32_t)min(c.pages - 1, (int64_t)0x7FFFFFFF));
        const uint8_t *codes = c.k_codes + kv_head(c, page, h, S) + (int64_t)(pos & ((1 << c.page_log2) - 1)) * S;
        for (int i = 0; i < s.n; ++i) {
            const KvSeen x = kv_seen(a, s, i);
            if (pos < x.lo || pos >= x.hi) continue;
            for (int g = 0; g < a.group; ++g) {
                const float lse = w.lse[(int64_t)(s.t0 + i) * c.heads * a.group + h * a.group + g];
                if (lse == -INFINITY) continue;
                const uint16_t *q = a.q + (s.t0 + i) * a.q_token + (h * a.group + g) * a.q_head;
                float dot = 0.f;
                for (int n = 0; n < S; ++n) {
                    const int code = codes[n];
                    if (code >= c.K) continue;
                    float k[SUB], v[SUB];
                    kv_unpack<FP16>(kv_load<SUB>(c.k_centres + ((int64_t)(h * S + n) * c.K + code) * SUB), k);
                    kv_unpack<FP16>(kv_load<SUB>(q + n * SUB), v);
                    for (int e = 0; e < SUB; ++e) dot = __builtin_fmaf(k[e], v[e], dot);
                }
                float z = a.cap_log2 > 0.f ? kv_capped(dot * a.scale_cap, a.cap_log2) : dot * a.scale_log2;
                if (a.slopes) z -= a.slopes[h * a.group + g] * kLog2e * (float)abs(x.at - pos);
                sum += __builtin_amdgcn_exp2f(z - lse * kLog2e);
            }
        }
    }
    *to = w.add ? *to + sum : sum;
}

template <int SUB>
hipError_t launch(const KvCache &c, const KvNew &n, const KvWeigh &w, hipStream_t s)
{
    const int64_t chunks = (w.positions + kThreads - 1) / kThreads;
    const auto kernel = c.fp16 ? kv_weigh_kernel<SUB, true> : kv_weigh_kernel<SUB, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(chunks * c.heads * n.seqs)), dim3(kThreads), 0, s, c, n, w, (int)chunks);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_weigh(const KvCache &c, const KvNew &n, const KvWeigh &w, hipStream_t s)
{
    return c.sub == 2 ? launch<2>(c, n, w, s) : c.sub == 4 ? launch<4>(c, n, w, s) : launch<8>(c, n, w, s);
}

}  // namespace lloyd
