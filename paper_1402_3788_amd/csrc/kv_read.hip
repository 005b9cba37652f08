// Reading keys and values back from the cache: the centres that the codes name.
#include "kv_device.h"

namespace lloyd {

namespace {

constexpr int kThreads = 256;

// One sub-vector of one head of one token, key and value, to a thread.
template <int SUB>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache c, KvTokens t, int64_t units)
{
    const int S = c.dim / SUB, kinds = c.heads * S;
    for (int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x; u < units;
         u += (int64_t)gridDim.x * kThreads) {
        const int64_t tok = u / kinds;
        const int kind = (int)(u - tok * kinds), h = kind / S, s = kind - h * S;
        int64_t page;
        int off;
        KvEntry<SUB> k{}, v{};
        if (kv_slot(c, t.slots[tok], &page, &off)) {
            const int64_t head = (page * c.heads + h) << c.page_log2;
            const int kc = c.k_codes[(head + off) * S + s];
            const int vc = c.v_codes[head * S + ((int64_t)s << c.page_log2) + off];
            if (kc < c.K) k = kv_load<SUB>(c.k_centres + ((int64_t)kind * c.K + kc) * SUB);
            if (vc < c.K) v = kv_load<SUB>(c.v_centres + ((int64_t)kind * c.K + vc) * SUB);
        }
        *reinterpret_cast<KvEntry<SUB> *>(t.k + tok * t.k_token + h * t.k_head + s * SUB) = k;
        *reinterpret_cast<KvEntry<SUB> *>(t.v + tok * t.v_token + h * t.v_head + s * SUB) = v;
    }
}

template <int SUB>
hipError_t launch(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    const int64_t units = t.tokens * c.heads * (c.dim / SUB);
    const int64_t groups = (units + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((kv_read_kernel<SUB>), dim3((unsigned)(groups < 65536 ? groups : 65536)),
                       dim3(kThreads), 0, s, c, t, units);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_read(const KvCache &c, const KvTokens &t, hipStream_t s)
{
    return c.sub == 2 ? launch<2>(c, t, s) : c.sub == 4 ? launch<4>(c, t, s) : launch<8>(c, t, s);
}

}  // namespace lloyd
