// The key-value cache in K-means codes: what kv_api.hip hands to the kernels of
// kv_write.hip, kv_read.hip and kv_attend.hip.
#pragma once

#include "lloyd.h"

namespace lloyd {

constexpr int kKvMaxSeqs = 4096;
constexpr int kKvMaxGroup = 128;     // query heads of one key-value head
constexpr int kKvTile = 32;          // positions of one step of a wave's attention
constexpr int kKvQueries = 16;       // query heads of one workgroup (columns of an MFMA)

// Wavefronts of an attention workgroup.
constexpr int kv_waves(int dim) { return dim == 64 ? 16 : 12; }

// The cache as the caller describes it (kmeans_kv_t, checked).
struct KvCache {
    const uint16_t *k_centres, *v_centres;
    uint8_t *k_codes, *v_codes;
    int64_t pages;
    int page_log2;
    int heads, dim, sub, K;
    bool fp16;
};

struct KvTokens {
    const int64_t *slots;
    int64_t tokens;
    uint16_t *k, *v;                 // read from by the encoder, written by the reader
    int64_t k_token, k_head, v_token, v_head;
};

// The sequence that begins in a workgroup's share of the tiles and ends in
// another's (b < 0: there is none), and the workgroups that have a part of it.
struct KvShared {
    int32_t b, parts;
};

struct KvAttend {
    const uint16_t *q;
    int64_t q_seq, q_head;
    int seqs, group;                 // group: query heads of one key-value head
    const int32_t *table;
    int64_t table_stride;
    int table_pages;
    const int32_t *lengths, *starts;
    float scale_log2;                // scale * log2(e)
    uint16_t *out;
    int64_t out_seq, out_head;
    float *lse;
    // workspace
    KvShared *shared;                // [workgroups]
    float *part_o, *part_ml;
};

// Launch geometry of the attention (pure host code).
struct KvAttendPlan {
    int splits;                      // workgroups of one head and block of queries
    int qblocks;                     // blocks of kKvQueries query heads
    size_t shared_off, part_o_off, part_ml_off, total;   // workspace
};

KvAttendPlan plan_kv_attend(const KvCache &c, int seqs, int group, int64_t table_pages);

hipError_t launch_kv_write(const KvCache &c, const KvTokens &t, hipStream_t s);
hipError_t launch_kv_read(const KvCache &c, const KvTokens &t, hipStream_t s);
hipError_t launch_kv_attend(const KvCache &c, const KvAttend &a, const KvAttendPlan &p,
                            hipStream_t s);

}  // namespace lloyd
