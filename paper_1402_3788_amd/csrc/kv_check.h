// Host checks that the key-value cache's C entry points share.
#pragma once

#include "../../include/kmeans.h"
#include "kv.h"

namespace lloyd {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline bool good_strides(int64_t outer, int64_t head)
{
    return outer >= 0 && head >= 0 && outer % 8 == 0 && head % 8 == 0;
}

// Everything of the description but its pointers.
inline int check_shape(const kmeans_kv_t *kv)
{
    if (!kv) return KMEANS_EINVAL;
    if (kv->pages < 1 || kv->page < 1 || kv->heads < 1 || kv->dim < 1 || kv->sub < 1 || kv->K < 1)
        return KMEANS_EINVAL;
    if (kv->type != KMEANS_KV_BF16 && kv->type != KMEANS_KV_FP16) return KMEANS_EINVAL;
    if (kv->page < 8 || kv->page > 1024 || (kv->page & (kv->page - 1))) return KMEANS_EUNSUPPORTED;
    if (kv->pages >= (int64_t)1 << 31 || kv->heads > 1024 || kv->K > 256)
        return KMEANS_EUNSUPPORTED;
    if (kv->dim != 64 && kv->dim != 96 && kv->dim != 128) return KMEANS_EUNSUPPORTED;
    if (kv->sub != 2 && kv->sub != 4 && kv->sub != 8) return KMEANS_EUNSUPPORTED;
    return KMEANS_OK;
}

inline int check_cache(const kmeans_kv_t *kv)
{
    const int rc = check_shape(kv);
    if (rc) return rc;
    if (!kv->k_centres || !kv->v_centres || !kv->k_codes || !kv->v_codes) return KMEANS_EINVAL;
    if (!aligned16(kv->k_centres) || !aligned16(kv->v_centres) || !aligned16(kv->k_codes) ||
        !aligned16(kv->v_codes))
        return KMEANS_EINVAL;
    return KMEANS_OK;
}

inline KvCache cache_of(const kmeans_kv_t *kv)
{
    KvCache c{};
    c.k_centres = static_cast<const uint16_t *>(kv->k_centres);
    c.v_centres = static_cast<const uint16_t *>(kv->v_centres);
    c.k_codes = kv->k_codes;
    c.v_codes = kv->v_codes;
    c.pages = kv->pages;
    c.page_log2 = __builtin_ctz((unsigned)kv->page);
    c.heads = kv->heads;
    c.dim = kv->dim;
    c.sub = kv->sub;
    c.K = kv->K;
    c.fp16 = kv->type == KMEANS_KV_FP16;
    return c;
}

inline int hip_status(hipError_t e) { return e == hipSuccess ? KMEANS_OK : KMEANS_EHIP; }

}  // namespace lloyd
