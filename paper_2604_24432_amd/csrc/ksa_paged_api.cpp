// C-ABI entry points of the paged cache.  Every argument check happens before the first HIP call.
#include <algorithm>
#include <cmath>

#include "ksa_internal.h"
#include "ksa_paged.h"

namespace {

bool aligned(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// augmented rows of a chunk; one that is longer than every text may exceed 32 bits
int64_t chunk_rows(const ksa_params *p) { return (int64_t)p->chunk_len + p->n_summary; }
int64_t augmented(const ksa_params *p) {
    return (p->n_text / p->chunk_len) * chunk_rows(p) + p->n_text % p->chunk_len;
}

int check_sizes(const ksa_params *p, int64_t total_rows) {
    const int rc = ksa_validate_params(p);
    if (rc != KSA_OK) return rc;
    if (total_rows < 0) return KSA_ERR_INVALID_ARG;
    if (total_rows >= ((int64_t)1 << 31) / p->n_q_heads) return KSA_ERR_UNSUPPORTED;   // (row, head) pairs are int32 on the device
    return KSA_OK;
}

// The cache and the batch of a call, checked, with defaults filled in.
int check_call(KsaPagedCall &c, const ksa_params *p, const ksa_paged_cache *cache, const int32_t *cu_rows, const int32_t *start, int64_t total_rows) {
    const int rc = check_sizes(p, total_rows);
    if (rc != KSA_OK) return rc;
    if (!cache || !cu_rows || !start || !aligned(cu_rows, 4) || !aligned(start, 4)) return KSA_ERR_INVALID_ARG;
    const bool f8 = cache->format == KSA_CACHE_FP8;
    if ((!f8 && cache->format != KSA_CACHE_BF16) || cache->reserved != 0) return KSA_ERR_INVALID_ARG;
    const int32_t rows = cache->page_rows;
    if (rows < 8 || rows > 1024 || (rows & (rows - 1)) || cache->n_pages <= 0) return KSA_ERR_INVALID_ARG;
    if (cache->text_pages <= 0 || !cache->text_table || !aligned(cache->text_table, 4)) return KSA_ERR_INVALID_ARG;
    if (p->n_summary > 0 && (cache->summary_pages <= 0 || !cache->summary_table)) return KSA_ERR_INVALID_ARG;
    if (cache->summary_pages < 0 || !aligned(cache->summary_table, 4)) return KSA_ERR_INVALID_ARG;
    if (!cache->k || !cache->v || !aligned(cache->k, 16) || !aligned(cache->v, 16)) return KSA_ERR_INVALID_ARG;
    if (f8 != (cache->k_exp != nullptr) || f8 != (cache->v_exp != nullptr)) return KSA_ERR_INVALID_ARG;
    const int64_t *s = cache->strides, size = f8 ? 1 : 2;
    if (s[0] == 0 && s[1] == 0 && s[2] == 0) {
        c.cache_strides[2] = p->head_dim * size;
        c.cache_strides[1] = rows * c.cache_strides[2];
        c.cache_strides[0] = p->n_kv_heads * c.cache_strides[1];
    } else {
        for (int x = 0; x < 3; ++x) {
            if (s[x] <= 0 || s[x] > INT64_MAX / 2 || (s[x] * size) % 16 != 0) return KSA_ERR_INVALID_ARG;
            c.cache_strides[x] = s[x] * size;
        }
    }
    c.p = *p, c.cache = *cache;
    if (c.p.softmax_scale <= 0.f) c.p.softmax_scale = 1.0f / __builtin_sqrtf((float)p->head_dim);
    c.page_shift = __builtin_ctz((unsigned)rows);
    c.aug_len = (int32_t)augmented(p);
    c.cu_rows = cu_rows, c.start = start, c.total_rows = (int32_t)total_rows;
    return KSA_OK;
}

// {row, head} strides in elements of a [rows, heads, head_dim] bf16 tensor
int check_strides(int64_t out[2], const int64_t *given, int32_t heads, int32_t head_dim) {
    out[0] = given ? given[0] : (int64_t)heads * head_dim, out[1] = given ? given[1] : head_dim;
    return out[0] > 0 && out[1] > 0 && out[0] % 8 == 0 && out[1] % 8 == 0 ? KSA_OK : KSA_ERR_INVALID_ARG;
}

// Keys that so many consecutive rows of a sequence see together, none less: the summaries, the text of the window and of the rows.
int64_t most_keys(const ksa_params *p, int64_t rows) {
    const int64_t text = std::min<int64_t>(p->n_text, (int64_t)p->window_chunks * p->chunk_len + p->chunk_len + rows);
    return (int64_t)(p->n_text / p->chunk_len) * p->n_summary + text;
}

/*
 * How a call is dealt.  All times in us; spans: time.
 *
 * Few rows: a workgroup per sequence, KV head and span of the keys, about 512 of them (two on each compute unit), and no span below 128 keys, 256
 * from 64 sequences x KV heads on, 512 from 128 on; below 512 keys one span.
 *   sequences x KV heads   keys                   measured
 *                      1    400                   1: 7.9    4: 7.5
 *                      1    700                   1: 9.6    4: 7.8    6: 7.9
 *                      1   1200                   2: 11.1   6: 8.1   16: 8.5
 *                      1   9000                  16: 15.5  32: 12.9  64: 11.9
 *                      8   6000                   8: 17.3  24: 12.7  64: 13.1
 *                     32    800                   4: 11.0   8: 10.4  16: 10.9
 *                     32   4200                   4: 21.5   8: 17.6  16: 17.2  32: 21.9
 *                     64    800                   3: 12.8   4: 12.0   6: 13.7
 *                     64   1500                   4: 15.8   6: 16.4
 *                    128   9000, 8 rows, 8-bit    2: 78.5   4: 53.1   8: 52.3  16: 58.1
 *                    160    800                   1: 13.6   3: 15.0
 *                    256   1500, 4 rows, 8-bit    1: 26.2   2: 27.0
 *                    256   4000                   1: 57.6   2: 57.2   4: 55.9
 *                    512  16500                   1: 636    2: 641    4: 656
 *                     16  65536, 8 rows           8: 99    16: 89    32: 91
 * Spans dealt by the sequences' lengths (lengths 1 : 4) instead of the same number each: 57.4 and 53.8 with 128, 248 and 249 with 512.
 *
 * Many rows: tiles of 128 pairs, two on a compute unit; of 128, alone, whose two groups of waves have half of the keys each; of 256, alone, which take
 * their keys from memory half as often.  The kind and the spans are chosen by what they are expected to take: a start and an end, the key tiles of
 * a span one after the other, rounds where there are more workgroups than places, and for the records of several spans a second kernel.  Per key
 * tile of head_dim 128: 128 pairs 1.5 alone on a unit, 1.95 in pairs, two groups 1.0, 256 pairs 1.75.
 *                                                            128 pairs            two groups     256 pairs
 *   full attention, 64K keys, 32/8 heads, 2048 rows          1: 2292                             1: 2067
 *                                          512 rows          4: 614   8: 649      2: 603 4: 637  3: 620  4: 562  8: 591
 *   summaries, 4700 keys, 512 rows                           1: 99    4: 57       1: 75  2: 54   3: 60   4: 54
 *   2000 keys, 2304 rows                                     1: 58    2: 84       1: 72          1: 69
 *   10000 keys, 2048 rows                                    1: 294               1: 304         1: 269  2: 296
 *   4200 keys, 8 x 100 rows                                  1: 91    4: 47 6: 51 1: 69  2: 47   3: 57
 *   window of 1023, 16/16 heads, 1280 rows                   1: 39    3: 36       1: 34  2: 50   3: 38
 *   2700 keys, 2595 rows of six, 12/4 heads, head_dim 64     1: 52    2: 41       1: 41          3: 48
 *   830 keys, 64 rows, 8/4 heads                             1: 20    6: 12.3     6: 13.3        6: 13.5
 * Over twelve such calls what is chosen takes 1.4 % longer than the best of the three kinds with 1, 2, 3, 4, 6, 8 and 12 spans; without the second
 * kind 3 %.
 *
 * most: what is chosen here has at most so many spans.
 */
constexpr int64_t MOST_SPANS = 64;
KsaPagedPlan plan_paged(const ksa_params *p, int64_t total_rows, int64_t max_rows, int32_t n_splits, int64_t most = MOST_SPANS) {
    const int32_t group = p->n_q_heads / p->n_kv_heads;
    KsaPagedPlan plan = {false, n_splits, 0, 0, 0};
    if (max_rows * group <= KSA_PAGED_FEW) {
        plan.few = true;
        const int64_t units = (int64_t)p->batch * p->n_kv_heads;
        if (n_splits != 0) return plan;
        const int64_t keys = most_keys(p, max_rows);
        const int64_t least = units >= 128 ? 512 : units >= 64 ? 256 : 128;
        plan.n_splits = keys < 512 ? 1 : (int32_t)std::max<int64_t>(1, std::min({512 / units, keys / least, most}));
        return plan;
    }
    const double size = p->head_dim == 128 ? 1.0 : 0.7;
    const double records = 1.35e-6 * (double)total_rows * p->n_q_heads * ksa_paged_record(p->head_dim);   // written and read, of one span
    double best = 0;
    struct Kind {
        int32_t pairs, groups;
        double start, tile;   // a workgroup's start and end, a tile of keys
    };
    for (const Kind &kind : {Kind{128, 1, 3, 1.5}, Kind{128, 2, 6.5, 1.0}, Kind{256, 1, 6, 1.75}}) {
        // every sequence ends one tile of text and one of summaries before it is full; the latter's lists are short
        const int32_t pairs = kind.pairs;
        const int64_t slots = total_rows * group / pairs + (p->n_summary > 0 ? 2 : 1) * (int64_t)p->batch;
        const double rows = (double)total_rows * p->chunk_len / chunk_rows(p);
        const double full = rows * group / pairs, units = (p->batch == 1 ? std::ceil(full) : full + 0.5 * p->batch) * p->n_kv_heads;
        const int64_t tiles = (most_keys(p, std::min<int64_t>(max_rows, pairs / group + 1)) + 63) / 64;
        for (int32_t n = n_splits == 0 ? 1 : n_splits; n <= (n_splits == 0 ? most : n_splits); ++n) {
            if (n_splits == 0 && n > 1 && n > tiles) break;
            const bool two = pairs == 128 && kind.groups == 1;   // on a compute unit
            const double places = two ? 512 : 256, wgs = units * n;
            const double tile = size * (kind.tile + (two ? 0.45 * std::min(std::max((wgs - 256) / 256, 0.0), 1.0) : 0));
            const double rounds = std::max(1.0, 1.1 * wgs / places);   // (workgroups of different lengths)
            const double time = rounds * (kind.start + (double)((tiles + n - 1) / n) * tile) + (n > 1 ? 5 + records * n : 0);
            if (plan.slots == 0 || time < best) best = time, plan.pairs = pairs, plan.groups = kind.groups, plan.slots = (int32_t)slots, plan.n_splits = n;
        }
    }
    return plan;
}

bool bad_fwd(int64_t max_rows, int32_t n_splits) { return max_rows <= 0 || n_splits < 0 || n_splits > 1024; }

constexpr int64_t MOST_LANES = (int64_t)1 << 32;   // of a grid, none of its dimensions more

bool too_large(const ksa_params *p, int64_t total_rows, const KsaPagedPlan &plan) {
    if (plan.n_splits > 1 && total_rows * p->n_q_heads * (plan.n_splits > 8 ? 256 : 64) >= MOST_LANES) return true;
    return !plan.few && (int64_t)plan.slots * plan.n_splits * p->n_kv_heads * plan.pairs * 2 * plan.groups >= MOST_LANES;
}

size_t span_bytes(const ksa_params *p, int64_t total_rows) { return (size_t)total_rows * p->n_q_heads * ksa_paged_record(p->head_dim) * sizeof(float); }
size_t workspace_of(const ksa_params *p, int64_t total_rows, const KsaPagedPlan &plan) {
    return plan.n_splits == 1 ? 0 : plan.n_splits * span_bytes(p, total_rows);
}

int move_call(KsaPagedMove &a, const ksa_params *p, const ksa_paged_cache *cache, const void *k, const void *v, const int64_t *strides,
              const int32_t *cu_rows, const int32_t *start, int64_t total_rows) {
    const int rc = check_call(a.call, p, cache, cu_rows, start, total_rows);
    if (rc != KSA_OK) return rc;
    if (total_rows > 0 && (!k || !v)) return KSA_ERR_INVALID_ARG;
    if (!aligned(k, 16) || !aligned(v, 16)) return KSA_ERR_INVALID_ARG;
    if ((total_rows * p->head_dim / 2048 + 1) * p->n_kv_heads * 256 >= MOST_LANES) return KSA_ERR_UNSUPPORTED;
    return check_strides(a.strides, strides, p->n_kv_heads, p->head_dim);
}

}  // namespace

extern "C" {

int ksa_paged_pages(const ksa_params *p, int32_t page_rows, int64_t n_rows, int64_t *text_pages, int64_t *summary_pages) {
    const int rc = ksa_validate_params(p);
    if (rc != KSA_OK) return rc;
    if (page_rows < 8 || page_rows > 1024 || (page_rows & (page_rows - 1)) || n_rows < 0) return KSA_ERR_INVALID_ARG;
    if (n_rows > augmented(p)) return KSA_ERR_OUT_OF_RANGE;
    const int64_t w = chunk_rows(p), text = n_rows / w * p->chunk_len + std::min<int64_t>(n_rows % w, p->chunk_len);
    if (text_pages) *text_pages = (text + page_rows - 1) / page_rows;
    if (summary_pages) *summary_pages = (n_rows - text + page_rows - 1) / page_rows;
    return KSA_OK;
}

int ksa_paged_append(const ksa_params *p, const ksa_paged_cache *cache, const void *k_new, const void *v_new, const int64_t kv_strides[2],
                     const int32_t *cu_rows, const int32_t *start, int64_t total_rows, void *stream) {
    KsaPagedMove a;
    const int rc = move_call(a, p, cache, k_new, v_new, kv_strides, cu_rows, start, total_rows);
    if (rc != KSA_OK || total_rows == 0) return rc;
    a.k = const_cast<void *>(k_new), a.v = const_cast<void *>(v_new);   // (read only)
    return ksa_launch_paged_append(a, stream);
}

int ksa_paged_read(const ksa_params *p, const ksa_paged_cache *cache, void *k, void *v, const int64_t kv_strides[2], const int32_t *cu_rows,
                   const int32_t *start, int64_t total_rows, void *stream) {
    KsaPagedMove a;
    const int rc = move_call(a, p, cache, k, v, kv_strides, cu_rows, start, total_rows);
    if (rc != KSA_OK || total_rows == 0) return rc;
    a.k = k, a.v = v;
    return ksa_launch_paged_read(a, stream);
}

size_t ksa_paged_workspace_bytes(const ksa_params *p, int64_t total_rows, int64_t max_rows, int32_t n_splits) {
    if (check_sizes(p, total_rows) != KSA_OK || bad_fwd(max_rows, n_splits) || total_rows == 0) return 0;
    return workspace_of(p, total_rows, plan_paged(p, total_rows, std::min(max_rows, total_rows), n_splits));
}

int ksa_paged_fwd(const ksa_params *p, const ksa_paged_cache *cache, const void *q, void *o, float *lse, const int64_t q_strides[2],
                  const int64_t o_strides[2], const int32_t *cu_rows, const int32_t *start, int64_t total_rows, int64_t max_rows,
                  void *workspace, size_t workspace_bytes, int32_t n_splits, void *stream) {
    KsaPagedFwd a;
    int rc = check_call(a.call, p, cache, cu_rows, start, total_rows);
    if (rc != KSA_OK) return rc;
    if (bad_fwd(max_rows, n_splits)) return KSA_ERR_INVALID_ARG;
    if (total_rows > 0 && (!q || !o)) return KSA_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4) || !aligned(workspace, 16)) return KSA_ERR_INVALID_ARG;
    if ((rc = check_strides(a.q_strides, q_strides, p->n_q_heads, p->head_dim)) != KSA_OK) return rc;
    if ((rc = check_strides(a.o_strides, o_strides, p->n_q_heads, p->head_dim)) != KSA_OK) return rc;
    if (total_rows == 0) return KSA_OK;
    a.max_rows = (int32_t)std::min(max_rows, total_rows);
    const size_t room = std::min<size_t>(workspace_bytes / span_bytes(p, total_rows), MOST_SPANS);
    a.plan = plan_paged(p, total_rows, a.max_rows, n_splits, std::max<int64_t>(room, 1));
    if (too_large(p, total_rows, a.plan)) return KSA_ERR_UNSUPPORTED;
    const size_t need = workspace_of(p, total_rows, a.plan);
    if (need > 0 && !workspace) return KSA_ERR_INVALID_ARG;
    if (workspace_bytes < need) return KSA_ERR_WORKSPACE_TOO_SMALL;
    a.q = q, a.o = o, a.lse = lse, a.workspace = static_cast<float *>(workspace);
    return ksa_launch_paged_fwd(a, stream);
}

}  // extern "C"
