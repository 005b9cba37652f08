// C entry points of serving from the key-value cache: checks on the host, then the
// launches of kv_rotate.hip, kv_tokens.hip, kv_weigh.hip and kv_evict.hip.
#include "kv_check.h"
#include "kv_tokens.h"

#include <float.h>
#include <math.h>

using namespace lloyd;

namespace {

// |stride| of a row of outputs or inputs that are not 16-bit rows
bool good_rows(int64_t seq, int64_t head) { return seq >= 0 && head >= 0; }

int check_table(const kmeans_kv_t *kv, int32_t seqs, int64_t table_pages, int64_t table_stride)
{
    if (seqs < 0 || table_pages < 1 || table_stride < 0) return KMEANS_EINVAL;
    if (seqs > kKvMaxSeqs || table_pages > ((int64_t)1 << 30) / kv->page ||
        (int64_t)seqs * kv->heads >= (int64_t)1 << 18)
        return KMEANS_EUNSUPPORTED;
    return KMEANS_OK;
}

// Everything of the new tokens but their pointers.
int check_new(const kmeans_kv_t *kv, const kmeans_kv_tokens_t *t)
{
    if (!t) return KMEANS_EINVAL;
    const int rc = check_table(kv, t->seqs, t->table_pages, t->table_stride);
    if (rc) return rc;
    if (t->tokens < 0 || t->window < 0 || t->q_heads < 1 || t->q_heads % kv->heads != 0)
        return KMEANS_EINVAL;
    if (t->q_heads / kv->heads > kKvMaxGroup || t->tokens >= (int64_t)1 << 30 ||
        t->tokens * t->q_heads >= (int64_t)1 << 30 ||
        (t->seqs + t->tokens * (t->q_heads / kv->heads) / kKvRows) *
                (t->table_pages * kv->page / kKvTile + 2) >= (int64_t)1 << 27)
        return KMEANS_EUNSUPPORTED;
    if (!isfinite(t->scale * kLog2e) || !(t->cap >= 0.f) || !isfinite(2.f * (t->cap * kLog2e)))
        return KMEANS_EINVAL;
    const float x = t->cap > 0.f ? t->scale / t->cap : 0.f;
    if (!isfinite(x) || (t->scale != 0.f && t->cap > 0.f && fabsf(x) < FLT_MIN)) return KMEANS_EINVAL;
    return KMEANS_OK;
}

int check_new_pointers(const kmeans_kv_tokens_t *t, const void *q, int64_t q_token, int64_t q_head)
{
    if (!t->bounds || !t->table || !t->lengths) return KMEANS_EINVAL;
    if (t->tokens > 0 && (!q || !aligned16(q))) return KMEANS_EINVAL;
    return good_strides(q_token, q_head) ? KMEANS_OK : KMEANS_EINVAL;
}

KvNew new_of(const kmeans_kv_t *kv, const kmeans_kv_tokens_t *t, const void *q, int64_t q_token,
             int64_t q_head)
{
    KvNew n{};
    n.q = static_cast<const uint16_t *>(q);
    n.q_token = q_token;
    n.q_head = q_head;
    n.bounds = t->bounds;
    n.table = t->table;
    n.table_stride = t->table_stride;
    n.lengths = t->lengths;
    n.starts = t->starts;
    n.prefixes = t->prefixes;
    n.slopes = t->slopes;
    n.tokens = t->tokens;
    n.table_pages = (int)t->table_pages;
    n.seqs = t->seqs;
    n.group = t->q_heads / kv->heads;
    // no position is so far from another
    n.window = t->window >= 1 << 30 ? 0 : t->window;
    n.scale_log2 = t->scale * kLog2e;
    n.cap_log2 = t->cap * kLog2e;
    n.scale_cap = t->cap > 0.f ? t->scale / t->cap : 0.f;
    return n;
}

int check_turned(const KvTurned &x)
{
    if (x.heads == 0) return KMEANS_OK;
    if (x.heads < 0 || !x.from || !x.to || !aligned16(x.from) || !aligned16(x.to))
        return KMEANS_EINVAL;
    if (!good_strides(x.from_token, x.from_head) || !good_strides(x.to_token, x.to_head))
        return KMEANS_EINVAL;
    if (x.from == x.to && (x.from_token != x.to_token || x.from_head != x.to_head))
        return KMEANS_EINVAL;
    return x.heads > 4096 ? KMEANS_EUNSUPPORTED : KMEANS_OK;
}

}  // namespace

extern "C" {

int kmeans_kv_rotate(const kmeans_kv_turn_t *turn, const void *q, int64_t q_token, int64_t q_head,
                     int32_t q_heads, void *q_out, int64_t q_out_token, int64_t q_out_head,
                     const void *k, int64_t k_token, int64_t k_head, int32_t k_heads, void *k_out,
                     int64_t k_out_token, int64_t k_out_head, void *stream)
{
    if (!turn || turn->tokens < 0 || turn->dim < 1 || turn->half < 0 || !isfinite(turn->amplitude))
        return KMEANS_EINVAL;
    if (turn->type != KMEANS_KV_BF16 && turn->type != KMEANS_KV_FP16) return KMEANS_EINVAL;
    if (turn->flags & ~(KMEANS_KV_INTERLEAVED | KMEANS_KV_INVERSE)) return KMEANS_EINVAL;
    if (2 * (int64_t)turn->half > turn->dim) return KMEANS_EINVAL;
    if (turn->dim % 8 != 0 || turn->dim > 512 || turn->tokens >= (int64_t)1 << 31)
        return KMEANS_EUNSUPPORTED;
    KvRotate r{};
    r.positions = turn->positions;
    r.frequencies = turn->frequencies;
    r.tokens = turn->tokens;
    r.dim = turn->dim;
    r.half = turn->half;
    r.amplitude = turn->amplitude;
    r.fp16 = turn->type == KMEANS_KV_FP16;
    r.interleaved = turn->flags & KMEANS_KV_INTERLEAVED;
    r.inverse = turn->flags & KMEANS_KV_INVERSE;
    r.x[0] = KvTurned{static_cast<const uint16_t *>(q), static_cast<uint16_t *>(q_out), q_token,
                      q_head, q_out_token, q_out_head, q_heads};
    r.x[1] = KvTurned{static_cast<const uint16_t *>(k), static_cast<uint16_t *>(k_out), k_token,
                      k_head, k_out_token, k_out_head, k_heads};
    if (r.tokens == 0 || q_heads + (int64_t)k_heads == 0)
        return q_heads < 0 || k_heads < 0 ? KMEANS_EINVAL : KMEANS_OK;
    int rc = check_turned(r.x[0]);
    if (rc || (rc = check_turned(r.x[1]))) return rc;
    if (r.half > 0 && (!r.positions || !r.frequencies)) return KMEANS_EINVAL;
    return hip_status(launch_kv_rotate(r, static_cast<hipStream_t>(stream)));
}

size_t kmeans_kv_attend_tokens_workspace_bytes(const kmeans_kv_t *kv, const kmeans_kv_tokens_t *t)
{
    if (check_shape(kv) != KMEANS_OK || check_new(kv, t) != KMEANS_OK) return 0;
    return kv_attend_tokens_bytes(cache_of(kv), new_of(kv, t, nullptr, 0, 0));
}

int kmeans_kv_attend_tokens(const kmeans_kv_t *kv, const kmeans_kv_tokens_t *t, const void *q,
                            int64_t q_token, int64_t q_head, void *out, int64_t out_token,
                            int64_t out_head, float *lse, void *workspace, size_t workspace_bytes,
                            void *stream)
{
    int rc = check_cache(kv);
    if (rc || (rc = check_new(kv, t))) return rc;
    if (t->seqs == 0 || t->tokens == 0) return KMEANS_OK;
    if ((rc = check_new_pointers(t, q, q_token, q_head))) return rc;
    if (!out || !aligned16(out) || !good_strides(out_token, out_head)) return KMEANS_EINVAL;
    const KvCache c = cache_of(kv);
    const KvNew n = new_of(kv, t, q, q_token, q_head);
    if (!workspace || !aligned16(workspace) || workspace_bytes < kv_attend_tokens_bytes(c, n))
        return KMEANS_EWORKSPACE;
    const KvTokensOut o{static_cast<uint16_t *>(out), out_token, out_head, lse};
    return hip_status(launch_kv_attend_tokens(c, n, o, workspace, static_cast<hipStream_t>(stream)));
}

int kmeans_kv_weigh(const kmeans_kv_t *kv, const kmeans_kv_tokens_t *t, const void *q,
                    int64_t q_token, int64_t q_head, const float *lse, float *weights,
                    int64_t weights_seq, int64_t weights_head, int64_t positions, int32_t add,
                    void *stream)
{
    int rc = check_cache(kv);
    if (rc || (rc = check_new(kv, t))) return rc;
    if (positions < 0 || (add != 0 && add != 1)) return KMEANS_EINVAL;
    if (positions > (int64_t)1 << 30) return KMEANS_EUNSUPPORTED;
    if (t->seqs == 0 || positions == 0 || (add && t->tokens == 0)) return KMEANS_OK;
    if ((rc = check_new_pointers(t, q, q_token, q_head))) return rc;
    if (!weights || !good_rows(weights_seq, weights_head) || (t->tokens > 0 && !lse))
        return KMEANS_EINVAL;
    const KvWeigh w{lse, weights, weights_seq, weights_head, positions, add != 0};
    return hip_status(launch_kv_weigh(cache_of(kv), new_of(kv, t, q, q_token, q_head), w,
                                      static_cast<hipStream_t>(stream)));
}

int kmeans_kv_evict(const kmeans_kv_t *kv, const kmeans_kv_evict_t *e, int32_t *kept,
                    int32_t *lengths_out, float *weights_out, int64_t out_seq, int64_t out_head,
                    void *stream)
{
    int rc = check_cache(kv);
    if (rc) return rc;
    if (!e) return KMEANS_EINVAL;
    if ((rc = check_table(kv, e->seqs, e->table_pages, e->table_stride))) return rc;
    if (e->keep < 1 || e->recent < 0 || e->first < 0 || e->positions < 0 ||
        e->recent > e->keep - e->first)
        return KMEANS_EINVAL;
    if (e->positions > (int64_t)1 << 30 || e->keep > 1 << 30) return KMEANS_EUNSUPPORTED;
    if (e->to) {
        rc = check_table(kv, e->seqs, e->to_pages, e->to_stride);
        if (rc) return rc;
        const int64_t most = e->table_pages * kv->page;
        if (e->to_pages * kv->page < (e->keep < most ? e->keep : most)) return KMEANS_EINVAL;
    }
    if (e->seqs == 0) return KMEANS_OK;
    if (!e->table || !e->lengths || !kept || !lengths_out) return KMEANS_EINVAL;
    if (e->positions > 0 && (!e->weights || !weights_out)) return KMEANS_EINVAL;
    if (!good_rows(e->weights_seq, e->weights_head) || !good_rows(out_seq, out_head))
        return KMEANS_EINVAL;
    if (weights_out == e->weights && (out_seq != e->weights_seq || out_head != e->weights_head))
        return KMEANS_EINVAL;
    KvEvict x{};
    x.table = e->table;
    x.table_stride = e->table_stride;
    x.table_pages = (int)e->table_pages;
    x.lengths = e->lengths;
    x.weights = e->weights;
    x.weights_seq = e->weights_seq;
    x.weights_head = e->weights_head;
    x.positions = e->positions;
    x.seqs = e->seqs;
    x.keep = e->keep;
    x.recent = e->recent;
    x.first = e->first;
    x.in_place = e->to == nullptr;
    x.weights_in_place = weights_out == e->weights;
    x.to = e->to ? e->to : e->table;
    x.to_stride = e->to ? e->to_stride : e->table_stride;
    x.to_pages = (int)(e->to ? e->to_pages : e->table_pages);
    x.kept = kept;
    x.lengths_out = lengths_out;
    x.weights_out = weights_out;
    x.out_seq = out_seq;
    x.out_head = out_head;
    return hip_status(launch_kv_evict(cache_of(kv), x, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
