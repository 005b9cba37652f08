// Serving from the key-value cache: what kv_serve_api.hip hands to the kernels of
// kv_rotate.hip, kv_tokens.hip, kv_weigh.hip and kv_evict.hip.
#pragma once

#include "kv.h"

namespace lloyd {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr int kKvRows = 256;         // rows (query heads of new tokens) of a unit of attention

// One tensor [tokens][heads][dim] that is turned, and where to.
struct KvTurned {
    const uint16_t *from;
    uint16_t *to;
    int64_t from_token, from_head, to_token, to_head;
    int heads;
};

struct KvRotate {
    const int64_t *positions;
    const double *frequencies;
    int64_t tokens;
    int dim, half;
    float amplitude;
    bool fp16, interleaved, inverse;
    KvTurned x[2];                   // queries, keys
};

// New tokens and how they score cached positions (kmeans_kv_tokens_t, checked).
struct KvNew {
    const uint16_t *q;
    int64_t q_token, q_head;
    const int32_t *bounds, *table;
    int64_t table_stride;
    const int32_t *lengths, *starts, *prefixes;
    const float *slopes;
    int64_t tokens;
    int table_pages, seqs, group;    // group: query heads of one key-value head
    int window;                      // 0: none
    float scale_log2;                // scale * log2(e)
    float cap_log2, scale_cap;       // cap * log2(e) and scale / cap; cap_log2 0: no cap
};

struct KvTokensOut {
    uint16_t *out;
    int64_t out_token, out_head;
    float *lse;
};

struct KvWeigh {
    const float *lse;
    float *weights;
    int64_t weights_seq, weights_head, positions;
    bool add;
};

struct KvEvict {
    const int32_t *table;
    int64_t table_stride;
    int table_pages;
    const int32_t *lengths;
    const float *weights;
    int64_t weights_seq, weights_head, positions;
    int seqs, keep, recent, first;
    const int32_t *to;               // the table itself: in place
    int64_t to_stride;
    int to_pages;
    bool in_place;                   // codes
    bool weights_in_place;           // whether codes are or not
    int32_t *kept, *lengths_out;
    float *weights_out;
    int64_t out_seq, out_head;
};

hipError_t launch_kv_rotate(const KvRotate &r, hipStream_t s);
size_t kv_attend_tokens_bytes(const KvCache &c, const KvNew &n);
hipError_t launch_kv_attend_tokens(const KvCache &c, const KvNew &n, const KvTokensOut &o, void *ws,
                                   hipStream_t s);
hipError_t launch_kv_weigh(const KvCache &c, const KvNew &n, const KvWeigh &w, hipStream_t s);
hipError_t launch_kv_evict(const KvCache &c, const KvEvict &e, hipStream_t s);

}  // namespace lloyd
