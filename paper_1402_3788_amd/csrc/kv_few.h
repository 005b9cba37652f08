// Few new tokens of every sequence: what the attention of one new token (kv_attend.hip)
// takes in the place of its sequences.
#pragma once

#include "kv_tokens_device.h"

namespace lloyd {

// Units of `rows` rows of a call at most, which there is room for. Bounds that descend can
// make more of the same tokens: then there are none.
__host__ __device__ inline int64_t kv_most_units(const KvNew &n, int rows)
{
    return n.seqs + n.tokens * n.group / rows;
}

// Query heads of new tokens (rows) of a unit.
constexpr int kv_few_rows(bool wide) { return wide ? 16 : 8; }
constexpr int kKvMaxFew = 4096;      // units at most
// Tiles that are worth a workgroup of their own, where all are more than one's waves: what waves
// hold of a unit is joined one unit after the other, so that few to a workgroup are soon done.
// In us with 12 (a tile to a wave), 4, 2 and 1: 22, 15, 11, 13 (11 sequences of 54, 3 tokens of 4
// heads, 7 key heads), 17, 14, 11, 12 (7 of 32, 2 of 5, 3 key heads), 18.3, 14.6, 14.1, 13.6 (8 of
// 80, 4 of 4, 8 key heads), 14.7, 13.1, 13.2, 15.4 (one of 800, one of 4); longer ones have more
// tiles than all workgroups' waves and take what they took.
constexpr int kFewShare = 2;

struct KvFew : KvNew {
    uint16_t *out;
    int64_t out_token, out_head;
    float *lse;
    KvUnits units;
    int rows;                        // of a unit
    bool in_lanes;                   // up to 64 units: each workgroup works them out, one writes them
    // workspace
    KvShared *shared;
    float *part_o, *part_ml;
};

struct KvFewPlan {
    bool wide;
    int splits;                      // workgroups of a head
    int units;                       // at most
    bool in_lanes;                   // up to 64 sequences and units: no launch that works them out
    size_t total;                    // workspace
};

KvFewPlan plan_kv_few(const KvCache &c, const KvNew &n);
hipError_t launch_kv_few(const KvCache &c, const KvNew &n, const KvTokensOut &o, const KvFewPlan &p,
                         void *ws, hipStream_t s);

// Writes the units of `rows` rows of a call.
hipError_t launch_kv_units(const KvCache &c, const KvNew &n, const KvUnits &to, int rows, hipStream_t s);

}  // namespace lloyd
