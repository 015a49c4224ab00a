// Argument checks that the entry points of the paged cache share.  Every one of them happens before the first HIP call.
#ifndef KSA_PAGED_CHECKS_H_
#define KSA_PAGED_CHECKS_H_

#include <cmath>

#include "ksa_internal.h"
#include "ksa_paged.h"

namespace {

inline bool aligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// augmented rows of a chunk; one that is longer than every text may exceed 32 bits
inline int64_t chunk_rows(const ksa_params *p) { return (int64_t)p->chunk_len + p->n_summary; }
inline int64_t augmented(const ksa_params *p) {
    return (p->n_text / p->chunk_len) * chunk_rows(p) + p->n_text % p->chunk_len;
}

inline int check_sizes(const ksa_params *p, int64_t total_rows) {
    const int rc = ksa_validate_params(p);
    if (rc != KSA_OK) return rc;
    if (total_rows < 0) return KSA_ERR_INVALID_ARG;
    if (total_rows >= ((int64_t)1 << 31) / p->n_q_heads) return KSA_ERR_UNSUPPORTED;   // (row, head) pairs are int32 on the device
    return KSA_OK;
}

// The cache of a call, checked, with defaults filled in.
inline int check_cache(KsaPagedCall &c, const ksa_params *p, const ksa_paged_cache *cache) {
    if (!cache) return KSA_ERR_INVALID_ARG;
    if (cache->format < KSA_CACHE_BF16 || cache->format > KSA_CACHE_FP4 || cache->reserved != 0) return KSA_ERR_INVALID_ARG;
    const bool exps = cache->format != KSA_CACHE_BF16, f4 = cache->format == KSA_CACHE_FP4;
    const int32_t rows = cache->page_rows;
    if (rows < 8 || rows > 1024 || (rows & (rows - 1)) || cache->n_pages <= 0) return KSA_ERR_INVALID_ARG;
    if (cache->text_pages <= 0 || !cache->text_table || !aligned(cache->text_table, 4)) return KSA_ERR_INVALID_ARG;
    if (p->n_summary > 0 && (cache->summary_pages <= 0 || !cache->summary_table)) return KSA_ERR_INVALID_ARG;
    if (cache->summary_pages < 0 || !aligned(cache->summary_table, 4)) return KSA_ERR_INVALID_ARG;
    if (!cache->k || !cache->v || !aligned(cache->k, 16) || !aligned(cache->v, 16)) return KSA_ERR_INVALID_ARG;
    if (exps != (cache->k_exp != nullptr) || exps != (cache->v_exp != nullptr)) return KSA_ERR_INVALID_ARG;
    if (f4 && (!aligned(cache->k_exp, 4) || !aligned(cache->v_exp, 4))) return KSA_ERR_INVALID_ARG;   // (so that a row's bytes may be loaded together; no kernel does yet)
    const int64_t *s = cache->strides, size = exps ? 1 : 2;   // (of two elements in the 4-bit format)
    if (s[0] == 0 && s[1] == 0 && s[2] == 0) {
        c.cache_strides[2] = f4 ? p->head_dim / 2 : p->head_dim * size;
        c.cache_strides[1] = rows * c.cache_strides[2];
        c.cache_strides[0] = p->n_kv_heads * c.cache_strides[1];
    } else {
        for (int x = 0; x < 3; ++x) {
            if (s[x] <= 0 || s[x] > INT64_MAX / 2 || (s[x] * size) % 16 != 0) return KSA_ERR_INVALID_ARG;
            c.cache_strides[x] = s[x] * size;
        }
    }
    if (f4 && (c.cache_strides[0] > UINT32_MAX || c.cache_strides[2] > UINT32_MAX / rows)) return KSA_ERR_UNSUPPORTED;   // (places in a page are 32 bits)
    c.p = *p, c.cache = *cache;
    if (c.p.softmax_scale <= 0.f) c.p.softmax_scale = 1.0f / __builtin_sqrtf((float)p->head_dim);
    c.page_shift = __builtin_ctz((unsigned)rows);
    c.aug_len = (int32_t)augmented(p);
    return KSA_OK;
}

// ... and its batch.
inline int check_call(KsaPagedCall &c, const ksa_params *p, const ksa_paged_cache *cache, const int32_t *cu_rows, const int32_t *start, int64_t total_rows) {
    const int rc = check_sizes(p, total_rows);
    if (rc != KSA_OK) return rc;
    if (!cu_rows || !start || !aligned(cu_rows, 4) || !aligned(start, 4)) return KSA_ERR_INVALID_ARG;
    c.cu_rows = cu_rows, c.start = start, c.total_rows = (int32_t)total_rows;
    return check_cache(c, p, cache);
}

// {row, head} strides in elements of a [rows, heads, head_dim] bf16 tensor
inline int check_strides(int64_t out[2], const int64_t *given, int32_t heads, int32_t head_dim) {
    out[0] = given ? given[0] : (int64_t)heads * head_dim, out[1] = given ? given[1] : head_dim;
    return out[0] > 0 && out[1] > 0 && out[0] % 8 == 0 && out[1] % 8 == 0 ? KSA_OK : KSA_ERR_INVALID_ARG;
}

constexpr int64_t MOST_LANES = (int64_t)1 << 32;   // of a grid, none of its dimensions more
// A launch with a wave per row, four to a workgroup: 2^26 - 4 rows are the most.
inline bool too_many_waves(int64_t rows) { return (rows + 3) / 4 * 256 >= MOST_LANES; }

inline int move_call(KsaPagedMove &a, const ksa_params *p, const ksa_paged_cache *cache, const void *k, const void *v, const int64_t *strides,
              const int32_t *cu_rows, const int32_t *start, int64_t total_rows) {
    const int rc = check_call(a.call, p, cache, cu_rows, start, total_rows);
    if (rc != KSA_OK) return rc;
    if (total_rows > 0 && (!k || !v)) return KSA_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16)) return KSA_ERR_INVALID_ARG;
    if ((total_rows * p->head_dim / 2048 + 1) * p->n_kv_heads * 256 >= MOST_LANES) return KSA_ERR_UNSUPPORTED;
    return check_strides(a.strides, strides, p->n_kv_heads, p->head_dim);
}

}  // namespace

#endif
