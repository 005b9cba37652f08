// Encoding of keys and values into the cache: every sub-vector gets the number
// of its nearest centre (Eq. (2)).
#include "kv_device.h"

namespace lloyd {

namespace {

constexpr int kThreads = 256;

// A workgroup takes one sub-vector of one head of the keys or the values (its
// centres in LDS) for 256 tokens, one to a thread.
template <int SUB, bool FP16>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache c, KvTokens t, int64_t units)
{
    __shared__ KvEntry<SUB> book[256];
    const int S = c.dim / SUB, kinds = 2 * c.heads * S;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int kind = (int)(u % kinds);
        const int s = kind % S, h = kind / S % c.heads;
        const bool values = kind / S >= c.heads;
        const uint16_t *centres = (values ? c.v_centres : c.k_centres) +
                                  ((int64_t)h * S + s) * c.K * SUB;
        __syncthreads();
        for (int j = threadIdx.x; j < c.K; j += kThreads) book[j] = kv_load<SUB>(centres + j * SUB);
        __syncthreads();
        const int64_t tok = u / kinds * kThreads + threadIdx.x;
        int64_t page;
        int off;
        if (tok >= t.tokens || !kv_slot(c, t.slots[tok], &page, &off)) continue;
        const uint16_t *src = values ? t.v + tok * t.v_token + h * t.v_head
                                     : t.k + tok * t.k_token + h * t.k_head;
        float x[SUB];
        kv_unpack<FP16>(kv_load<SUB>(src + s * SUB), x);
        float best = INFINITY;
        int code = 0;
        for (int j = 0; j < c.K; ++j) {
            float y[SUB];
            kv_unpack<FP16>(book[j], y);
            const float d = kv_distance(x, y);
            if (d < best) { best = d; code = j; }
        }
        const int64_t head = (page * c.heads + h) << c.page_log2;
        if (values)
            c.v_codes[head * S + ((int64_t)s << c.page_log2) + off] = (uint8_t)code;
        else
            c.k_codes[(head + off) * S + s] = (uint8_t)code;
    }
}

template <int SUB>
hipError_t launch(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    const int64_t units = (t.tokens + kThreads - 1) / kThreads * (2 * c.heads * (c.dim / SUB));
    const unsigned grid = (unsigned)(units < 65536 ? units : 65536);
    if (c.fp16)
        hipLaunchKernelGGL((kv_write_kernel<SUB, true>), dim3(grid), dim3(kThreads), 0, s, c, t, units);
    else
        hipLaunchKernelGGL((kv_write_kernel<SUB, false>), dim3(grid), dim3(kThreads), 0, s, c, t, units);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_write(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    return c.sub == 2 ? launch<2>(c, t, s) : c.sub == 4 ? launch<4>(c, t, s) : launch<8>(c, t, s);
}

}  // namespace lloyd
