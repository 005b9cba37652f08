// C entry points of the key-value cache in K-means codes: checks on the host,
// then the launches of kv_write.hip, kv_read.hip and kv_attend.hip.
#include "../../include/kmeans.h"
#include "kv_check.h"

#include <math.h>

using namespace lloyd;

namespace {

int check_tokens(const KvTokens &t)
{
    if (t.tokens < 0) return KMEANS_EINVAL;
    if (t.tokens == 0) return KMEANS_OK;
    if (!t.slots || !t.k || !t.v || !aligned16(t.k) || !aligned16(t.v)) return KMEANS_EINVAL;
    if (!good_strides(t.k_token, t.k_head) || !good_strides(t.v_token, t.v_head))
        return KMEANS_EINVAL;
    if (t.tokens > ((int64_t)1 << 31) - 1) return KMEANS_EUNSUPPORTED;
    return KMEANS_OK;
}

int check_attend(const kmeans_kv_t *kv, int32_t seqs, int32_t q_heads, int64_t table_pages)
{
    if (seqs < 0 || q_heads < 1 || q_heads % kv->heads != 0 || table_pages < 1)
        return KMEANS_EINVAL;
    if (seqs > kKvMaxSeqs || q_heads / kv->heads > kKvMaxGroup ||
        table_pages > ((int64_t)1 << 30) / kv->page)
        return KMEANS_EUNSUPPORTED;
    // tiles of all sequences, workgroups of the joining launch
    if (seqs * ((table_pages * kv->page + kKvTile - 1) / kKvTile) >= (int64_t)1 << 31 ||
        (int64_t)seqs * q_heads >= (int64_t)1 << 24)
        return KMEANS_EUNSUPPORTED;
    return KMEANS_OK;
}

}  // namespace

extern "C" {

int kmeans_kv_write(const kmeans_kv_t *kv, const void *k, int64_t k_token, int64_t k_head,
                    const void *v, int64_t v_token, int64_t v_head, const int64_t *slots,
                    int64_t tokens, void *stream)
{
    int rc = check_cache(kv);
    if (rc) return rc;
    const KvTokens t{slots, tokens, const_cast<uint16_t *>(static_cast<const uint16_t *>(k)),
                     const_cast<uint16_t *>(static_cast<const uint16_t *>(v)),
                     k_token, k_head, v_token, v_head};
    if ((rc = check_tokens(t)) || tokens == 0) return rc;
    return hip_status(launch_kv_write(cache_of(kv), t, static_cast<hipStream_t>(stream)));
}

int kmeans_kv_read(const kmeans_kv_t *kv, const int64_t *slots, int64_t tokens, void *k,
                   int64_t k_token, int64_t k_head, void *v, int64_t v_token, int64_t v_head,
                   void *stream)
{
    int rc = check_cache(kv);
    if (rc) return rc;
    const KvTokens t{slots, tokens, static_cast<uint16_t *>(k), static_cast<uint16_t *>(v),
                     k_token, k_head, v_token, v_head};
    if ((rc = check_tokens(t)) || tokens == 0) return rc;
    return hip_status(launch_kv_read(cache_of(kv), t, static_cast<hipStream_t>(stream)));
}

size_t kmeans_kv_attend_workspace_bytes(const kmeans_kv_t *kv, int32_t seqs, int32_t q_heads,
                                        int64_t table_pages)
{
    if (check_shape(kv) != KMEANS_OK || check_attend(kv, seqs, q_heads, table_pages) != KMEANS_OK)
        return 0;
    return plan_kv_attend(cache_of(kv), seqs, q_heads / kv->heads, table_pages).total;
}

int kmeans_kv_attend(const kmeans_kv_t *kv, const void *q, int64_t q_seq, int64_t q_head,
                     int32_t seqs, int32_t q_heads, const int32_t *table, int64_t table_stride,
                     int64_t table_pages, const int32_t *lengths, const int32_t *starts,
                     float scale, void *out, int64_t out_seq, int64_t out_head, float *lse,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_cache(kv);
    if (rc || (rc = check_attend(kv, seqs, q_heads, table_pages))) return rc;
    const float scale_log2 = scale * 1.44269504088896341f;
    if (!isfinite(scale_log2)) return KMEANS_EINVAL;
    if (seqs == 0) return KMEANS_OK;
    if (!q || !out || !table || !lengths || !aligned16(q) || !aligned16(out))
        return KMEANS_EINVAL;
    if (!good_strides(q_seq, q_head) || !good_strides(out_seq, out_head) || table_stride < 0)
        return KMEANS_EINVAL;
    const KvCache c = cache_of(kv);
    const KvAttendPlan p = plan_kv_attend(c, seqs, q_heads / kv->heads, table_pages);
    if (!workspace || !aligned16(workspace) || workspace_bytes < p.total)
        return KMEANS_EWORKSPACE;
    char *ws = static_cast<char *>(workspace);
    KvAttend a{};
    a.q = static_cast<const uint16_t *>(q);
    a.q_seq = q_seq;
    a.q_head = q_head;
    a.seqs = seqs;
    a.group = q_heads / kv->heads;
    a.table = table;
    a.table_stride = table_stride;
    a.table_pages = (int)table_pages;
    a.lengths = lengths;
    a.starts = starts;
    a.scale_log2 = scale_log2;
    a.out = static_cast<uint16_t *>(out);
    a.out_seq = out_seq;
    a.out_head = out_head;
    a.lse = lse;
    a.shared = reinterpret_cast<KvShared *>(ws + p.shared_off);
    a.part_o = reinterpret_cast<float *>(ws + p.part_o_off);
    a.part_ml = reinterpret_cast<float *>(ws + p.part_ml_off);
    return hip_status(launch_kv_attend(c, a, p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
