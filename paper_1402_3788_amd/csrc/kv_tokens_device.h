// Device helpers of the kernels that take many new tokens (kv_tokens.hip, kv_weigh.hip).
#pragma once

#include "kv_device.h"
#include "kv_tokens.h"

namespace lloyd {

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

__device__ inline KvSeen kv_seen(const KvNew &a, const KvSeq &s, int i)
{
    KvSeen x;
    x.at = s.len - s.n + i;
    x.hi = max(x.at + 1, s.prefix);
    x.lo = a.starts ? max(a.starts[s.t0 + i], 0) : 0;
    if (a.window) x.lo = max(x.lo, x.at - a.window + 1);
    if (x.lo >= x.hi) x.lo = x.hi = 0;
    return x;
}

// cap * tanh(z / cap) to base 2, of x = z / cap. tanh x = 1 - 2 / (1 + e^2x): off by
// 2^-23 of 1 for small x, where a cap of 50 makes it 4e-6 of a score.
__device__ inline float kv_capped(float x, float cap_log2)
{
    const float e = __builtin_amdgcn_exp2f(x * (2.f * kLog2e));
    return cap_log2 - 2.f * cap_log2 * __builtin_amdgcn_rcpf(1.f + e);
}

}  // namespace lloyd
