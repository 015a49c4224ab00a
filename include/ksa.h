/*
 * ksa.h -- C ABI of the MI355X (gfx950) Kwai Summary Attention hot path.
 *
 * The library computes  O = softmax(Q K^T * scale + M_KSA) V  (the KSA attention formula of the
 * paper's distillation section) over the augmented sequence of section 2.2.1 / Eq. 1, in which
 * n_summary summary tokens follow every chunk of chunk_len text tokens, with the visibility M_KSA
 * of section 2.2.2 / Eq. 3:
 *   - a text token in chunk j sees the text of chunks max(0, j - window_chunks) .. j up to itself,
 *     and the summary tokens of chunks 0 .. j - window_chunks - 1 (summaries of chunks still inside
 *     the window are not visible);
 *   - a summary token sees the text of its own chunk, itself, and the earlier summary tokens of
 *     its own chunk (KSA_FLAG_SUMMARY_SELF_ONLY drops the earlier siblings).
 * The paper has one summary token per chunk (n_summary = 1, chunk_len = k); n_summary > 1 with
 * compress_ratio = chunk_len / n_summary is this library's generalisation of it.
 *
 * Conventions
 *   - Plain C, no exceptions cross the boundary.  Every function returns a ksa_status (0 = OK).
 *   - "host" / "device" is stated for every pointer.  The caller owns every tensor and the stream;
 *     the library owns the opaque ksa_layout until ksa_layout_destroy.
 *   - Argument validation happens before any HIP call, so bad arguments are reported even on a
 *     machine without a GPU.  Inputs are never written.
 *   - Kernels are enqueued on the caller's HIP stream and are asynchronous; nothing synchronises.
 *   - Tensor element type is bf16 (q, k, v, o, caches); log-sum-exp outputs are fp32.
 *     Scores and accumulators are fp32; P is rounded to bf16 before the P V product in prefill.
 */
#ifndef KSA_H_
#define KSA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum ksa_status {
    KSA_OK = 0,
    KSA_ERR_INVALID_ARG = -1,        /* null pointer, non-positive size, inconsistent parameters, ... */
    KSA_ERR_UNSUPPORTED = -2,        /* head_dim / group size the kernels were not built for        */
    KSA_ERR_WORKSPACE_TOO_SMALL = -3,
    KSA_ERR_HIP = -4,                /* a HIP runtime call failed (no device, launch error, OOM)    */
    KSA_ERR_OUT_OF_RANGE = -5,       /* an index argument lies outside the layout                   */
    KSA_ERR_SCRATCH_LIMIT = -6,      /* the problem needs more than the library's static scratch buffer holds */
    KSA_ERR_OUT_OF_MEMORY = -7       /* a host allocation failed while building a layout            */
} ksa_status;

#define KSA_FLAG_SUMMARY_SELF_ONLY 1u /* summary rows see, among summaries, only themselves */

/* Problem statement, in the paper's terms (Eq. 1-3; Table "model_config"). */
typedef struct ksa_params {
    int32_t batch;           /* B                                                               */
    int32_t n_text;          /* n: text tokens per sequence (prefill); context capacity (decode) */
    int32_t chunk_len;       /* c: text tokens per chunk (an incomplete last chunk has no summaries) */
    int32_t n_summary;       /* m: summary tokens after each chunk (paper: 1); 0 = no summaries  */
    int32_t compress_ratio;  /* k = c / m; validated (k * m == c) when m > 0, ignored when m == 0 */
    int32_t window_chunks;   /* C >= 0: previous chunks whose text stays visible (Eq. 2 / Eq. 3)  */
    int32_t n_q_heads;       /* Hq, a multiple of n_kv_heads (GQA: query head h reads KV head h / (Hq/Hkv)) */
    int32_t n_kv_heads;      /* Hkv                                                              */
    int32_t head_dim;        /* d: 64 or 128                                                     */
    float softmax_scale;     /* <= 0 selects 1/sqrt(head_dim)                                    */
    uint32_t flags;          /* KSA_FLAG_*                                                       */
} ksa_params;

typedef struct ksa_layout ksa_layout;

/* Key-tile kinds reported by ksa_layout_tile_pairs. */
#define KSA_TILE_FULL 0    /* every (query row, key) pair of the tile pair is visible: no mask applied */
#define KSA_TILE_MASKED 1  /* per-element bounds are applied                                          */
/* Index spaces of a tile: compact text index i (0..n-1) or compact summary ordinal u (0..J*m-1). */
#define KSA_SPACE_TEXT 0
#define KSA_SPACE_SUMMARY 1

/*
 * ksa_build_layout: the integer side of Eq. 1 and Eq. 3 -- index maps of the augmented sequence,
 * per-row visible ranges, and the block-sparse schedule that lists, for every query tile, only the
 * key tiles that hold at least one visible pair (section 2.3: only non-zero block pairs are loaded).
 * Pure host work; touches no GPU.  *out (host) receives a new layout owned by the library.
 * Errors: INVALID_ARG for bad params (see ksa_params), UNSUPPORTED for head_dim not in {64, 128},
 * OUT_OF_MEMORY if the host cannot hold the schedule.
 */
int ksa_build_layout(const ksa_params *params /*host*/, ksa_layout **out /*host*/);
void ksa_layout_destroy(ksa_layout *layout);

/*
 * Copies the schedule to the current HIP device (one hipMalloc + one hipMemcpy).  ksa_prefill_fwd
 * does this itself on first use; calling it ahead keeps the first timed call allocation-free.  After it,
 * ksa_prefill_fwd and ksa_prefill_bwd enqueue kernels only (no allocation, memset or synchronisation) and may be
 * captured into a HIP graph.
 */
int ksa_layout_upload(ksa_layout *layout);

/* Rows of the augmented sequence (Eq. 1) of n_text text tokens under params' chunk_len and n_summary:
 * (n_text / c)(c + m) + n_text mod c (params->n_text itself is not used).  For sizing the q / k / v tensors. */
int ksa_augmented_rows(const ksa_params *params /*host*/, int64_t n_text, int64_t *rows /*host*/);

/* ---- introspection (host arrays, caller-allocated) used by the bit-exact layout tests ---------- */

/* L = (n/c) * (c+m) + n mod c augmented rows (an incomplete last chunk has text rows only), J = n/c whole chunks,
 * the query / key tile heights of the schedule, and the number of query heads (of one KV head) a prefill
 * workgroup handles together: 1, 2 or 4, with q_tile_rows * heads_per_workgroup = 256.  Any pointer may be NULL. */
int ksa_layout_dims(const ksa_layout *layout, int64_t *aug_len, int32_t *n_chunks, int32_t *q_tile_rows,
                    int32_t *k_tile_rows, int32_t *heads_per_workgroup);
/* Eq. 1 index maps.  aug_chunk, aug_is_summary, position_ids: [L]; text_to_aug: [n]; summary_to_aug: [J*m].
 * position_ids gives a summary token the position of its chunk's last text token (section 2.2.1).
 * Any pointer may be NULL to skip that array. */
int ksa_layout_index_maps(const ksa_layout *layout, int32_t *aug_chunk, uint8_t *aug_is_summary,
                          int32_t *position_ids, int32_t *text_to_aug, int32_t *summary_to_aug);
/* Visible ranges of augmented row aq: out = {summary_lo, summary_hi, text_lo, text_hi}: summary ordinals
 * [summary_lo, summary_hi) and text indices [text_lo, text_hi) are visible, nothing else. */
int ksa_layout_row_ranges(const ksa_layout *layout, int64_t aq, int32_t out[4]);
/* Row aq of M_KSA expanded from the row ranges: row_out[ak] = 1 iff visible, ak in [0, L). */
int ksa_layout_mask_row(const ksa_layout *layout, int64_t aq, uint8_t *row_out);
/*
 * The (query tile, key tile) pairs of the schedule, for one (batch, head): what the prefill kernel for long key runs
 * visits (the one for short runs and odd chunk shapes works its key lists out by itself).  Pass NULL arrays to
 * get *n_pairs only.  Pair x: query rows [q_begin[x], q_begin[x]+q_count[x]) of space q_space[x], key rows
 * [k_begin[x], k_begin[x]+k_count[x]) of space k_space[x], kind[x] = KSA_TILE_FULL or KSA_TILE_MASKED.
 */
int ksa_layout_tile_pairs(const ksa_layout *layout, int64_t *n_pairs, uint8_t *q_space, int32_t *q_begin,
                          int32_t *q_count, uint8_t *k_space, int32_t *k_begin, int32_t *k_count, uint8_t *kind);

/*
 * The launch order of the prefill kernel for long key runs: entry x is what workgroup x does -- the query tile (q_space[x], q_begin[x]) for
 * batch[x] and the query heads q_head[x] .. q_head[x] + heads_per_workgroup - 1 (ksa_layout_dims);
 * q_begin[x] = -1 marks a padding workgroup that does nothing.  Consecutive workgroup
 * ids are dealt to the 8 XCDs round-robin, so entries congruent mod 8 share an L2.  NULL arrays: count only.
 */
int ksa_layout_launch_order(const ksa_layout *layout, int64_t *n_entries, uint8_t *q_space, int32_t *q_begin,
                            int32_t *batch, int32_t *q_head);

/* ---- prefill ------------------------------------------------------------------------------------ */

/*
 * Bytes of device scratch memory ksa_prefill_fwd needs for this layout (0 for a NULL layout): room for a
 * key-major copy of V, batch * n_kv_heads * head_dim * (n_text + n_summary_tokens, each rounded up to 64) bf16,
 * followed by the largest squared K row norm per (batch, KV head, 64-key tile) and per (batch, KV head), fp32.
 */
size_t ksa_prefill_workspace_bytes(const ksa_layout *layout);

/*
 * ksa_prefill_fwd: attention output of all L augmented rows (text and summary rows alike),
 *   O = softmax(Q K^T * scale + M_KSA) V with the visibility of Eq. 3 over the sequence of Eq. 1.
 *   q [B, L, Hq, d], k and v [B, L, Hkv, d], o [B, L, Hq, d]: device, bf16, last dim contiguous;
 *   *_strides = {batch, row, head} strides in elements; NULL = contiguous in the order above.
 *   lse: device fp32 [B, Hq, L] contiguous, natural-log sum-exp of the scaled visible scores; may be NULL.
 *   workspace: device memory, 16-byte aligned, at least ksa_prefill_workspace_bytes(layout) bytes, owned by the
 *   caller, and needed until the work enqueued on `stream` has finished.  What the call writes there depends on the
 *   layout: a key-major copy of V and the largest K row norms (long key runs), the norms alone (short ones; of short texts
 *   only those per (batch, KV head)), or nothing (chunk shapes that are no powers of two).  From the norms the kernels derive a fixed softmax reference per row wherever
 *   |q| max |k| * scale is small enough to rule out overflow and underflow; other rows keep a running maximum.  Calls that
 *   share a workspace must be stream-ordered.
 *   stream: hipStream_t (NULL = default stream).
 * o may be the memory of q (same strides), or that of v where chunk_len and n_summary are powers of two; otherwise outputs
 * share no memory with inputs.
 * bf16 MFMA for Q K^T and P V over the live key tiles of every query tile, fp32 online softmax.
 * Value range: the weights of a row are kept within [2^-88, 2^32] relative to its reference and summed in fp32, so
 * the output is finite as long as max |v| times the number of visible keys stays below 2^95.
 * Errors: INVALID_ARG (null tensors or workspace, misaligned pointers: 16-byte alignment required),
 * WORKSPACE_TOO_SMALL, HIP.
 */
int ksa_prefill_fwd(ksa_layout *layout, const void *q, const void *k, const void *v, void *o, float *lse,
                    const int64_t q_strides[3], const int64_t kv_strides[3], const int64_t o_strides[3],
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * ksa_prefill_relayout_v: only the preparation pass of ksa_prefill_fwd, run on v alone: the key-major copy of V
 * goes into the workspace (same v, kv_strides, workspace and error rules as there), and the row-norm part of the pass
 * reads v in place of k (same shape, same cost; its result is not used by anything).  ksa_prefill_fwd always runs the
 * pass itself; this entry point exists so that the pass and the main kernel can be timed apart.
 */
int ksa_prefill_relayout_v(ksa_layout *layout, const void *v, const int64_t kv_strides[3], void *workspace,
                           size_t workspace_bytes, void *stream);

/* Bytes of device scratch memory ksa_prefill_bwd needs for this layout (0 for a NULL layout): two fp32 per
 * (batch, query head, row), the rows of each index space (text, summary) rounded up to a multiple of 64. */
size_t ksa_prefill_bwd_workspace_bytes(const ksa_layout *layout);

/*
 * ksa_prefill_bwd: gradients of ksa_prefill_fwd's output with respect to q, k and v for an upstream gradient
 * d_o = dLoss/dO (the paper's block-sparse kernel is its training kernel too, section 2.3, Kernel Design; the formulas are
 * the derivative of the attention definition):
 *   P = exp(Q K^T * scale - lse) on visible pairs (Eq. 3), dV = P^T dO, dS = P o (dO V^T - rowsum(dO o O)),
 *   dQ = scale * dS K, dK = scale * dS^T Q; with grouped heads a KV head sums over its query heads.
 *   q, k, v, o, lse: what ksa_prefill_fwd read and wrote (same shapes, o_strides for o AND d_o; lse is required);
 *   d_o [B, L, Hq, d], dq [B, L, Hq, d], dk and dv [B, L, Hkv, d]: device, bf16, last dim contiguous;
 *   dq_strides for dq, dkv_strides for dk and dv ({batch, row, head}, NULL = contiguous).  Every row of dq, dk
 *   and dv is written.
 *   workspace: device memory, 16-byte aligned, at least ksa_prefill_bwd_workspace_bytes(layout) bytes, owned by
 *   the caller, overwritten, needed until the work enqueued on `stream` has finished.
 * On short sequences several workgroups share a long key tile; their fp32 partial sums are kept in the memory of dq, which
 * is written last.  That takes a dense dq that shares no memory with another tensor of the call, and dk / dv that share none
 * with k / v; otherwise (a dq that is a view of a fused gradient tensor, say) no tile is shared, which is slower on short
 * sequences (head_dim 128, c 64, m 8; 2 x 4096 tokens, 32 / 8 heads: 377 -> 604 us; 16K tokens, 8 / 1 heads: 381 -> 3533).
 * No atomics: results do not depend on the launch order.  head_dim 64 or 128.  The row strides of q, k / v and d_o
 * must be positive, and the rows that 64 consecutive text (or summary) positions span in the augmented sequence must
 * lie within 4 GiB of each other in each of these tensors (a chunk_len of 4096 at a row stride of 8 KiB still does);
 * else UNSUPPORTED.
 * Errors: INVALID_ARG (null or misaligned pointers, bad strides), WORKSPACE_TOO_SMALL, UNSUPPORTED, HIP.
 */
int ksa_prefill_bwd(ksa_layout *layout, const void *q, const void *k, const void *v, const void *o, const float *lse,
                    const void *d_o, void *dq, void *dk, void *dv, const int64_t q_strides[3],
                    const int64_t kv_strides[3], const int64_t o_strides[3], const int64_t dq_strides[3],
                    const int64_t dkv_strides[3], void *workspace, size_t workspace_bytes, void *stream);

/* ---- decode over the summary KV cache (section 2.3.1) ------------------------------------------ */

/*
 * Cache geometry of this library (one K and one V tensor, device bf16, [B, Hkv, cache_rows, d]):
 *   rows [0, S_cap)                         Summary Token Buffer: summary ordinal u = j*m + slot at row u;
 *   rows [S_cap, S_cap + (C+1)*c)           text ring: text index i of chunk j = i / c at row
 *                                           S_cap + (j mod (C+1)) * c + i mod c.
 * S_cap = (n_text / c) * m.  The chunk being written overwrites, in place, the chunk that just left the
 * window, so no copy is needed when a chunk completes.  Summaries of in-window chunks are resident in the
 * buffer but are not read (Eq. 3).
 */
int ksa_cache_geometry(const ksa_params *params /*host*/, int32_t *summary_capacity, int32_t *cache_rows);
/* Cache row of text index i / of summary ordinal u (host helpers for packing a cache). */
int ksa_cache_text_row(const ksa_params *params, int64_t text_index, int32_t *row);
int ksa_cache_summary_row(const ksa_params *params, int64_t summary_ordinal, int32_t *row);
/*
 * Rows a new text token at text index pos reads: up to three (offset, length) row ranges, in the order
 * summaries, ring part 1, ring part 2; unused ranges have length 0.  out = {off0, len0, off1, len1, off2, len2}.
 */
int ksa_decode_ranges(const ksa_params *params /*host*/, int64_t pos, int32_t out[6]);

/* Bytes of device workspace ksa_decode_fwd needs for the given number of key splits (0 = library default). */
size_t ksa_decode_workspace_bytes(const ksa_params *params, int32_t n_splits);

/*
 * ksa_decode_fwd: one new text token per sequence.
 *   q [B, Hq, d] device bf16 contiguous; k_cache, v_cache device bf16 with cache_strides = {batch, head, row}
 *   in elements (NULL = contiguous [B, Hkv, cache_rows, d]); pos: device int32 [B], text index of the new
 *   token, whose K/V must already be in the cache; o [B, Hq, d] device bf16; lse device fp32 [B, Hq] or NULL.
 *   workspace: device, at least ksa_decode_workspace_bytes(params, n_splits).  n_splits = 0: the library chooses the number of
 *   spans, for large problems by each sequence's own length.
 * Split-K over the visible rows: each workgroup streams one span of K and V rows once for all Hq/Hkv query
 * heads of a KV head and writes a partial (max, sum, o); a second kernel merges the spans by log-sum-exp.
 * Sequences whose pos is outside [0, n_text) produce NaN rows (device-side positions cannot be validated
 * on the host without a synchronisation).
 */
int ksa_decode_fwd(const ksa_params *params /*host*/, const void *q, const void *k_cache, const void *v_cache,
                   const int32_t *pos, void *o, float *lse, const int64_t cache_strides[3], void *workspace,
                   size_t workspace_bytes, int32_t n_splits, void *stream);

/*
 * ksa_decode_fwd_static: ksa_decode_fwd for callers that cannot allocate device memory or hand over a workspace --
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, kernels and
 * results as ksa_decode_fwd (bit for bit, for the same n_splits), but the partial records of the spans live in a
 * static device array inside the library instead of a caller workspace; the call allocates and frees nothing.
 *   - Limit: ksa_decode_workspace_bytes(params, n_splits) must not exceed KSA_DECODE_STATIC_SCRATCH_BYTES (8 MiB;
 *     the 128K decode workload -- batch 64, 32 query heads, 3 spans -- needs 3.2 MB); otherwise the call returns
 *     KSA_ERR_SCRATCH_LIMIT and enqueues nothing.
 *   - Every GPU holds its own copy of the array for the life of the process; its address is looked up on the
 *     first call on that GPU (one hipGetSymbolAddress, no allocation).
 *   - All calls on one GPU share the array: calls on different streams that overlap in time race on it; calls must
 *     be stream-ordered or otherwise serialised by the caller.  The array keeps the previous call's records; every
 *     record the merge kernel reads is rewritten by the same call's first kernel, so nothing needs clearing.
 */
#define KSA_DECODE_STATIC_SCRATCH_BYTES (8u << 20)
int ksa_decode_fwd_static(const ksa_params *params /*host*/, const void *q, const void *k_cache, const void *v_cache,
                          const int32_t *pos, void *o, float *lse, const int64_t cache_strides[3], int32_t n_splits,
                          void *stream);

/* ---- cache lifecycle of the decode loop (section 2.3.1, the step-by-step cache description) ----------- */

/* Kind of a row / of a query in the calls below. */
#define KSA_ROW_TEXT 0     /* a text token; its position argument is a text index i in [0, n_text)            */
#define KSA_ROW_SUMMARY 1  /* a summary token; its position argument is a summary ordinal u = j*m + slot      */

/*
 * ksa_cache_from_prefill: hand-off from a prefilled sequence to the decode loop.  k, v: device bf16
 * [B, L, Hkv, d], the augmented sequence of n_prefill text tokens (at most params->n_text;
 * L = (n_prefill / c)(c + m) + n_prefill mod c), kv_strides = {batch, row, head} in elements (NULL = contiguous).
 * Writes, per (batch, KV head), the summaries of all n_prefill / c whole chunks into the Summary Token Buffer and
 * the text of the window into the text ring of k_cache, v_cache: the incomplete last chunk, if any, and the C whole
 * chunks before it; without an incomplete chunk the last min(n_prefill / c, C + 1) whole chunks (geometry above,
 * cache_strides = {batch, head, row}, NULL = contiguous).  Other cache rows are left as they are.  The next
 * token of every sequence is then text index n_prefill.  params->n_text is the capacity of the cache.
 * n_prefill = 0 is a no-op (k and v may be NULL then).
 * Errors: INVALID_ARG (null or misaligned pointers, negative n_prefill, strides not multiples of 8),
 * OUT_OF_RANGE (n_prefill > n_text), HIP.
 */
int ksa_cache_from_prefill(const ksa_params *params /*host*/, int64_t n_prefill, const void *k, const void *v,
                           const int64_t kv_strides[3], void *k_cache, void *v_cache,
                           const int64_t cache_strides[3], void *stream);

/*
 * ksa_cache_append: one new row per sequence.  k_new, v_new: device bf16 [B, Hkv, d] contiguous.
 * kind = KSA_ROW_TEXT: pos[b] (device int32 [B]) is the text index of the token; its row goes into the slot of the
 * current chunk in the ring, over the row of the chunk that left the window C + 1 chunks ago (the paper's insert
 * and evict steps in one store).  kind = KSA_ROW_SUMMARY: pos[b] is the summary ordinal j*m + slot; the row is
 * committed to the Summary Token Buffer (the paper's commit step).  A sequence whose pos is outside the cache
 * is skipped.  Errors: INVALID_ARG (null or misaligned pointers, unknown kind, kind = SUMMARY with m = 0), HIP.
 */
int ksa_cache_append(const ksa_params *params /*host*/, int32_t kind, const void *k_new, const void *v_new,
                     const int32_t *pos, void *k_cache, void *v_cache, const int64_t cache_strides[3],
                     void *stream);

/*
 * Rows a summary token with ordinal u = j*m + slot reads (Eq. 3, summary rows): the text of its own chunk j
 * (c ring rows) and the summaries of the same chunk up to itself (only itself with params->flags bit 0).
 * out = {off0, len0, off1, len1}: summary buffer range, ring range.
 */
int ksa_decode_summary_ranges(const ksa_params *params /*host*/, int64_t ordinal, int32_t out[4]);

/*
 * ksa_decode_summary_fwd: the summary-token step of the decode loop: one summary query per sequence, run when
 * a chunk has been completed.  Arguments as ksa_decode_fwd, except that ordinal[b] (device int32 [B]) is the
 * summary ordinal j*m + slot of the query; the K/V rows of the chunk's text and of the summary itself must be in
 * the cache (ksa_cache_append).  Same kernels as ksa_decode_fwd over at most c + m rows.
 */
int ksa_decode_summary_fwd(const ksa_params *params /*host*/, const void *q, const void *k_cache,
                           const void *v_cache, const int32_t *ordinal, void *o, float *lse,
                           const int64_t cache_strides[3], void *workspace, size_t workspace_bytes,
                           int32_t n_splits, void *stream);

/* ---- paged cache: many new rows per sequence, bf16, 8-bit or 4-bit floats ------------------------------------------- */

/*
 * A batch of augmented sequences (Eq. 1) whose K / V rows lie in pages of one pool.  A page is page_rows rows of every KV
 * head.  Text index i of sequence b lies in slot i mod page_rows of page text_table[b, i div page_rows], summary ordinal u in slot
 * u mod page_rows of page summary_table[b, u div page_rows].  Nothing else says where a row is: the two tables may name one page for
 * several sequences (a shared prompt), and a page that only holds text behind the window (Eq. 3) may be given to other
 * rows; its entry is then negative.  An entry outside [0, n_pages), and a row behind a table's last column, is no page: a row that
 * goes there is not written, is read back as NaN, and makes the outputs of the rows that see it NaN.  Entries that no row of the call lies
 * in or sees may hold anything.
 *
 * KSA_CACHE_FP8 holds a row of one KV head as 8-bit floats (e4m3: 4 significant bits, largest 448) times a power of two 2^e:
 * e is the least integer in [-117, 119] with max |x| <= 448 * 2^e over the row's finite elements (119 if none is), every element is x / 2^e rounded
 * to the nearest e4m3 number (ties to even; what lies beyond 448 * 2^119 = 2.98e38 becomes that), infinities and NaN become
 * NaN.  k_exp and v_exp hold e + 127.  With a byte there that is none of those (in a slot never written) the rows that see it may come out as
 * anything, and only they.  What a row stands for is zero or a normal bf16 number per element: reading it back and attending to it
 * add no rounding.
 *
 * KSA_CACHE_FP4 holds a row of one KV head in groups of 32 elements, each as 4-bit floats (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times
 * a power of two 2^e of the group's: e is the least integer in [-125, 125] with max |x| <= 7 * 2^e over the group (7, half way to the 8 that e2m1 lacks, and
 * what lies beyond become 6), every element is x / 2^e rounded to the nearest e2m1 number (ties to the even code).  Two elements are a byte, the one
 * with the even index in the low bits.  k_exp and v_exp hold e + 127 per group; 255 says that some element of the group was an infinity or NaN: then all
 * 32 are NaN.  Other bytes (in a slot never written) are as above.  Here too reading and attending add no rounding.
 */
#define KSA_CACHE_BF16 0
#define KSA_CACHE_FP8 1
#define KSA_CACHE_FP4 2
typedef struct ksa_paged_cache {
    int32_t format;                 /* KSA_CACHE_*                                                                     */
    int32_t page_rows;              /* rows per page: a power of two in [8, 1024]                                      */
    int32_t n_pages;                /* pages in the pool                                                               */
    int32_t text_pages;             /* columns of text_table                                                           */
    int32_t summary_pages;          /* columns of summary_table; 0 only if n_summary is 0                              */
    int32_t reserved;               /* 0                                                                               */
    const int32_t *text_table;      /* device [batch, text_pages]                                                      */
    const int32_t *summary_table;   /* device [batch, summary_pages]; may be NULL if n_summary is 0                    */
    void *k, *v;                    /* device, bf16, e4m3 or pairs of e2m1, [n_pages, Hkv, page_rows, d (pairs: d / 2)], last dim contiguous */
    uint8_t *k_exp, *v_exp;         /* device, contiguous: [n_pages, Hkv, page_rows] for KSA_CACHE_FP8, [n_pages, Hkv, page_rows, d / 32] (on 4 bytes)
                                       for KSA_CACHE_FP4, else NULL */
    int64_t strides[3];             /* of k and v: {page, head, row} in elements, multiples of 16 bytes; {0, 0, 0} = contiguous.  KSA_CACHE_FP4: in bytes;
                                       UNSUPPORTED if the page's, or page_rows times the row's, exceeds 2^32 - 1 */
} ksa_paged_cache;

/*
 * The calls below take a ragged batch of new rows, one behind the other in tensors of total_rows rows: rows
 * [cu_rows[b], cu_rows[b + 1]) (device int32 [batch + 1], not decreasing, within [0, total_rows]) belong to sequence b and are
 * its augmented rows start[b], start[b] + 1, ... (device int32 [batch]); a sequence may have none.  Rows of no sequence are
 * left as they are.  A sequence with start[b] < 0, with rows behind those of params->n_text text tokens (the capacity), or
 * whose two entries of cu_rows lie outside [0, total_rows] is out of place: ksa_paged_append skips it, the other calls set its rows to NaN.
 * Nothing is allocated, cleared or waited for: all of them may be captured into a graph, and what lies in device memory (cu_rows,
 * start, the tables) may change between replays.  total_rows = 0 is a no-op.
 * kv_strides, q_strides, o_strides: {row, head} in elements, multiples of 8, the last dim contiguous; NULL = contiguous.
 * Errors of all: INVALID_ARG (null or misaligned pointers: 16 bytes, 4 for int32 and fp32; bad strides or cache fields), UNSUPPORTED (more
 * than a launch holds: 2^28 (row, KV head) pairs of head_dim 128 into or out of the cache, 2^31 (row, query head) pairs of the attention, 2^24 in several
 * spans; what ksa_params excludes), HIP.
 */

/* Columns that the tables need for the first n_rows augmented rows of a sequence.  Errors: INVALID_ARG, OUT_OF_RANGE (n_rows beyond the rows of
 * params->n_text text tokens). */
int ksa_paged_pages(const ksa_params *params /*host*/, int32_t page_rows, int64_t n_rows, int64_t *text_pages /*host*/,
                    int64_t *summary_pages /*host*/);

/*
 * ksa_paged_append: k_new, v_new (device bf16 [total_rows, Hkv, d]) go into the cache.  One call takes a step's token, a chunk
 * of a prompt or all of it (start[b] = 0: the k, v of ksa_prefill_fwd), text and summary rows alike.  Rows without a page are skipped.  If two rows of a
 * call go to one place, which of them is held afterwards is not said (and K may be the one's, V the other's).
 */
int ksa_paged_append(const ksa_params *params /*host*/, const ksa_paged_cache *cache /*host*/, const void *k_new, const void *v_new,
                     const int64_t kv_strides[2], const int32_t *cu_rows, const int32_t *start, int64_t total_rows, void *stream);

/* ksa_paged_read: the same rows back out of the cache, as bf16, into k, v (device [total_rows, Hkv, d]). */
int ksa_paged_read(const ksa_params *params /*host*/, const ksa_paged_cache *cache /*host*/, void *k, void *v,
                   const int64_t kv_strides[2], const int32_t *cu_rows, const int32_t *start, int64_t total_rows, void *stream);

/* Bytes of device workspace ksa_paged_fwd needs for total_rows new rows, at most max_rows of one sequence, and this number of key splits
 * (0 = library default, for which it is what the fastest number takes: few rows may take more than many, which are cut into fewer spans); 0 also
 * for arguments that make no sense. */
size_t ksa_paged_workspace_bytes(const ksa_params *params /*host*/, int64_t total_rows, int64_t max_rows, int32_t n_splits);

/*
 * ksa_paged_fwd: the new rows attend to what they see (Eq. 3), their own K / V rows included, which must be in the cache.  One row
 * per sequence is a decode step, of text or of a summary token; a few are drafted tokens checked in one pass; thousands are a
 * chunk of a prompt.  What a row's outputs are does not depend on how the rows before it were dealt to calls, apart from rounding.
 *   q, o: device bf16 [total_rows, Hq, d]; lse: device fp32 [total_rows, Hq] contiguous, natural-log sum-exp of the scaled
 *   visible scores, or NULL.  o may be the memory of q (same strides).
 *   max_rows: no sequence has more new rows; one that has is out of place.  It sizes the launch.
 *   workspace: device, 16-byte aligned, at least ksa_paged_workspace_bytes(params, total_rows, max_rows, n_splits) bytes (NULL if that is 0); with
 *   n_splits = 0 it may hold less (NULL and 0 bytes among it): the library then takes no more spans than it holds.  It is
 *   needed until the work enqueued on `stream` has finished; calls that share one must be stream-ordered.
 *   n_splits: spans that the keys of a sequence are cut into, each read by workgroups of its own; 0: the library chooses (by params->n_text,
 *   the context that it must reckon with, and the workspace), else 1 .. 1024.  Another number of them rounds differently.
 * Scores, maxima and sums are fp32; weights are rounded to bf16 for P V.  A row's outputs depend on nothing that it does not see:
 * infinities and NaN elsewhere do not reach it.  No atomics.
 * Errors also: WORKSPACE_TOO_SMALL.
 */
int ksa_paged_fwd(const ksa_params *params /*host*/, const ksa_paged_cache *cache /*host*/, const void *q, void *o, float *lse,
                  const int64_t q_strides[2], const int64_t o_strides[2], const int32_t *cu_rows, const int32_t *start,
                  int64_t total_rows, int64_t max_rows, void *workspace, size_t workspace_bytes, int32_t n_splits, void *stream);

/* ---- rotary positions ---------------------------------------------------------------------------------------------------- */

/*
 * Rotary positions turn pairs of a head's elements: (a, b) becomes magnitude * (a cos x - b sin x, b cos x + a sin x), x = position * f_i for pair i of dim / 2.
 * The pairs are (2i, 2i + 1) with `interleaved`, else (i, i + dim / 2); elements from `dim` on stay as they are.  A text row's position is its text
 * index, a summary row's that of its chunk's last text row (section 2.2.1, as ksa_layout_index_maps).  The caches take keys that have been turned.
 * Frequencies are in turns per position, as fractions of 2^64, so that the angle of any position is exact to 2^-32 of a turn.
 */
typedef struct ksa_rotary {
    int32_t dim;                    /* even, 2 .. head_dim                                    */
    int32_t interleaved;            /* 0 or 1                                                 */
    float magnitude;                /* finite, positive                                       */
    int32_t reserved;               /* 0                                                      */
    const uint64_t *turns;          /* device [dim / 2], 8-byte aligned (ksa_rotary_turns)    */
} ksa_rotary;

#define KSA_ROTARY_PLAIN 0          /* f_i = base^(-2i / dim) radians per position                                               */
#define KSA_ROTARY_LINEAR 1         /* f_i / factor                                                                             */
#define KSA_ROTARY_BY_PARTS 2       /* with r = original * f_i / 2 pi turns over the original context and s = (r - slow) / (fast - slow) kept within 0 .. 1:
                                       f_i (s + (1 - s) / factor); magnitude 0.1 ln(factor) + 1                                  */
typedef struct ksa_rotary_rule {
    int32_t dim, scaling;           /* scaling: KSA_ROTARY_*                                                                    */
    double base;                    /* more than 1                                                                              */
    double factor;                  /* at least 1; by how much the context has grown                                             */
    double original;                /* by parts: positions of the original context, more than 0                                 */
    double slow, fast;              /* by parts: 0 <= slow < fast                                                               */
} ksa_rotary_rule;

/* The frequencies of a rule (host array [dim / 2]) and its magnitude (host), for a ksa_rotary.  Errors: INVALID_ARG. */
int ksa_rotary_turns(const ksa_rotary_rule *rule /*host*/, uint64_t *turns /*host*/, float *magnitude /*host*/);

/*
 * ksa_rotary_fwd: rows of whole augmented sequences (those of params->n_text text tokens) are turned: q [B, L, Hq, d] into q_out, k [B, L, Hkv, d] into k_out,
 * device bf16, last dim contiguous.  q and q_out, or k and k_out, may be NULL.  An output may be the memory of its input (same strides).
 * *_strides = {batch, row, head} in elements, multiples of 8, positive; NULL = contiguous.  Angles and products are fp32, each output is rounded once.
 * ksa_rotary_bwd: gradients with respect to q and k from those with respect to what ksa_rotary_fwd gave: turned back, times magnitude.
 * Errors: INVALID_ARG (null or misaligned pointers: 16 bytes; bad strides or rotary fields), UNSUPPORTED (more than 2^26 - 4 rows of all sequences), HIP.
 */
int ksa_rotary_fwd(const ksa_params *params /*host*/, const ksa_rotary *rotary /*host*/, const void *q, const void *k, void *q_out, void *k_out,
                   const int64_t q_strides[3], const int64_t k_strides[3], const int64_t q_out_strides[3], const int64_t k_out_strides[3], void *stream);
int ksa_rotary_bwd(const ksa_params *params /*host*/, const ksa_rotary *rotary /*host*/, const void *dq_out, const void *dk_out, void *dq, void *dk,
                   const int64_t dq_out_strides[3], const int64_t dk_out_strides[3], const int64_t dq_strides[3], const int64_t dk_strides[3], void *stream);

/*
 * ksa_rotary_step: one new row per sequence of the decode loop (ksa_decode_fwd, ksa_cache_append): q [B, Hq, d] into q_out, k [B, Hkv, d] into k_out. kind and pos
 * (device int32 [B]) as in ksa_cache_append: text indices, or summary ordinals. Rows of a sequence whose pos is outside the text (its whole chunks' summaries) become NaN.
 * *_strides = {batch, head}; all else as ksa_rotary_fwd. Errors also: INVALID_ARG (unknown kind, kind = SUMMARY with m = 0, null or misaligned pos).
 */
int ksa_rotary_step(const ksa_params *params /*host*/, const ksa_rotary *rotary /*host*/, int32_t kind, const void *q, const void *k, const int32_t *pos, void *q_out,
                    void *k_out, const int64_t q_strides[2], const int64_t k_strides[2], const int64_t q_out_strides[2], const int64_t k_out_strides[2], void *stream);

/*
 * ksa_paged_rotary: a serving step's new rows in one launch: q (device bf16 [total_rows, Hq, d]) is turned into q_out, k_new is turned, and goes with v_new into the
 * cache, as ksa_paged_append puts it (k is rounded to bf16 in between: the same bits as in two steps).  Batch, tables, capacity and errors as there (and UNSUPPORTED
 * above 2^26 - 4 rows); rows of q of a sequence out of place become NaN in q_out.  q and q_out may be NULL; q_out may be the memory of q (same strides).
 */
int ksa_paged_rotary(const ksa_params *params /*host*/, const ksa_paged_cache *cache /*host*/, const ksa_rotary *rotary /*host*/, const void *q, void *q_out,
                     const void *k_new, const void *v_new, const int64_t q_strides[2], const int64_t q_out_strides[2], const int64_t kv_strides[2],
                     const int32_t *cu_rows, const int32_t *start, int64_t total_rows, void *stream);

/* ---- a step's rows and pages from the sequences' lengths --------------------------------------------------------------------- */

/*
 * ksa_paged_advance: what a step needs to know and to have, worked out on the device.  Sequence b holds held[b] text tokens (with the summaries of their
 * whole chunks) and gets new_text[b] more, whose rows (text, and the summaries of every chunk that they complete) are the step's new rows: start[b] and
 * cu_rows as the calls above take them.  new_text[b] < 0: the sequence has ended; it has no rows and gives all its pages back.  A sequence with held[b] < 0 or
 * held[b] + new_text[b] > params->n_text is out of place: start[b] = -1, it has no rows and its pages stay.
 *
 * Pages: page_refs (device int32 [n_pages]) counts how many table entries name a page (a shared prompt: several); a page with 0 is free.  The call
 *   - gives back (entry = -1, its page's count one less) text columns that only hold text which no row sees any more (Eq. 3 for a sequence that holds held[b]),
 *     and the columns of sequences that have ended,
 *   - gives a free page (entry = page, count 1) to every column that begins with or behind the first new row of its kind, holds a new row and has no page
 *     (an entry outside [0, n_pages)): the lowest free pages, in the order of sequences, text before summaries, columns ascending,
 * and leaves everything else, so a second call with the same lengths changes nothing.  A page must not take new rows while several entries name it: share whole pages.
 * *lacking is the number of columns that got no page because none was free; their rows are not stored and read as NaN until the sequence ends.
 * The cache's tables are written; k, v and the exponents are not looked at.
 *
 *   held, new_text: device int32 [batch]; cu_rows: device int32 [batch + 1]; start: device int32 [batch]; lacking: device int32 [1].
 *   Row maps of the step's rows, device [total_rows], each may be NULL: slots (int64): page * page_rows + slot, -1 without a page; positions (int32): as rotary
 *   positions take them; tokens (int32): the row's place among the new text tokens of all sequences, or -1 - s for the s-th summary of its chunk.  Rows behind the last
 *   sequence's get -1, 0 and -1.  total_rows may be less than the rows there are; it only says how long the maps are.
 *   workspace: device, 16-byte aligned, at least ksa_paged_advance_workspace_bytes bytes, needed until the work enqueued on `stream` has finished;
 *   calls that share one must be stream-ordered.
 * Counts beyond 2^31 - 1 (cu_rows) stay there.  Nothing is allocated, cleared or waited for; the call may be captured into a graph.  Results do not depend on the
 * order of execution.  Errors: INVALID_ARG, WORKSPACE_TOO_SMALL, UNSUPPORTED (2^31 - 4096 columns
 * of both tables over all sequences and more; total_rows of 2^31 - 256 and more), HIP.
 */
size_t ksa_paged_advance_workspace_bytes(const ksa_params *params /*host*/, const ksa_paged_cache *cache /*host*/);
int ksa_paged_advance(const ksa_params *params /*host*/, const ksa_paged_cache *cache /*host*/, int32_t *page_refs, const int32_t *held, const int32_t *new_text,
                      int32_t *cu_rows, int32_t *start, int32_t *lacking, int64_t *slots, int32_t *positions, int32_t *tokens, int64_t total_rows,
                      void *workspace, size_t workspace_bytes, void *stream);

const char *ksa_status_string(int status);
/* Static description of the build: tile sizes and the gfx target, e.g. for logs. */
const char *ksa_build_info(void);

#ifdef __cplusplus
}
#endif
#endif /* KSA_H_ */
