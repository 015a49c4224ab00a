// The paged cache's launches: what the argument checks hand to the kernels, and the device-side pieces that the kernels share.
#ifndef KSA_PAGED_H_
#define KSA_PAGED_H_

#include "ksa.h"

// A checked call on the paged cache.  Strides in bytes, defaults filled in.
struct KsaPagedCall {
    ksa_params p;
    ksa_paged_cache cache;
    int64_t cache_strides[3];     // {page, head, row}
    int32_t page_shift;
    int32_t aug_len;              // augmented rows of a sequence of params.n_text text tokens
    const int32_t *cu_rows, *start;
    int32_t total_rows;
};

// rows in (append) or out (read): k, v [total_rows, Hkv, d] bf16
struct KsaPagedMove {
    KsaPagedCall call;
    void *k, *v;
    int64_t strides[2];           // {row, head}
};
int ksa_launch_paged_append(const KsaPagedMove &a, void *stream);
int ksa_launch_paged_read(const KsaPagedMove &a, void *stream);
void ksa_launch_paged_append_fp4(const KsaPagedMove &a, void *stream);
void ksa_launch_paged_read_fp4(const KsaPagedMove &a, void *stream);

// ... turned on their way, and q with them (null: no q)
struct KsaPagedRotary {
    KsaPagedMove move;
    ksa_rotary rotary;
    const void *q;
    void *q_out;
    int64_t q_strides[2], out_strides[2];   // {row, head}
};
int ksa_launch_paged_rotary(const KsaPagedRotary &a, void *stream);

// a step's rows and pages
struct KsaPagedAdvance {
    KsaPagedCall call;
    int32_t *page_refs;
    const int32_t *held, *new_text;
    int32_t *cu_rows, *start, *lacking;
    int64_t *slots;
    int32_t *positions, *tokens;
    int32_t *workspace;
};
size_t ksa_paged_advance_ints(int32_t batch, int32_t n_pages);   // of the workspace
int ksa_launch_paged_advance(const KsaPagedAdvance &a, void *stream);

#define KSA_PAGED_FEW 32
// How the attention of a call is dealt to workgroups.
struct KsaPagedPlan {
    bool few;                     // the kernel for few rows: at most KSA_PAGED_FEW (row, query head) pairs of a sequence and KV head
    int32_t n_splits;             // spans of the keys
    int32_t pairs;                // many rows: (row, query head) pairs of a query tile, 128 or 256
    int32_t groups;               // ... of 128: groups of waves with a part of the keys each, 1 or 2
    int32_t slots;                // ... and query tiles of all sequences, none less
};
// Floats of a span's record for one (row, query head): the output, then maximum and sum (padded to 16 bytes)
inline int64_t ksa_paged_record(int32_t head_dim) { return head_dim + 4; }

struct KsaPagedFwd {
    KsaPagedCall call;
    KsaPagedPlan plan;
    const void *q;
    void *o;
    float *lse, *workspace;
    int64_t q_strides[2], o_strides[2];   // {row, head}
    int32_t max_rows;
};
int ksa_launch_paged_fwd(const KsaPagedFwd &a, void *stream);
void ksa_launch_paged_fwd_fp4(const KsaPagedFwd &a, void *stream);   // all but the join of spans

#ifdef __HIPCC__
#include "ksa_device.h"
#include "ksa_paged_index.h"

namespace {

inline PagedRows paged_rows(const KsaPagedCall &L) {
    PagedRows a;
    a.text_table = L.cache.text_table, a.sum_table = L.cache.summary_table;
    a.text_cols = L.cache.text_pages, a.sum_cols = L.p.n_summary > 0 ? L.cache.summary_pages : 0;
    a.n_pages = L.cache.n_pages, a.shift = L.page_shift;
    a.cu = L.cu_rows, a.start = L.start, a.batch = L.p.batch, a.total = L.total_rows, a.aug_len = L.aug_len;
    // (where no chunk is ever whole there are no summaries, and c + m, which may exceed 32 bits then, is c)
    a.c = L.p.chunk_len, a.m = L.p.chunk_len > L.p.n_text ? 0 : L.p.n_summary, a.C = L.p.window_chunks, a.self_only = (L.p.flags & KSA_FLAG_SUMMARY_SELF_ONLY) ? 1 : 0;
    a.by_w = ksa_divisor(a.c + a.m), a.by_c = ksa_divisor(a.c), a.by_m = ksa_divisor(a.m > 0 ? a.m : 1);
    return a;
}

// The new rows of a packed row's sequence, and the sequence; a.batch and none for a row behind them all.  A sequence is the row's if so many end at
// or in front of the row (cu_rows does not decrease).  The wave's rows are first (the same in all lanes) .. first + ROWS - 1; 64 sequences are
// looked at together, all that there is to know of them loaded at once.
template <int ROWS>
__device__ __forceinline__ NewRows sequence_of(const PagedRows &a, int first, int row, int max_rows, int &b) {
    const int lane = threadIdx.x & 63;
    for (b = 0; b < a.batch; b += 64) {
        const bool any = b + lane < a.batch;
        const NewRows s = new_rows(a, min(b + lane, a.batch - 1), max_rows);
        const int end = a.cu[min(b + lane, a.batch - 1) + 1];
        const uint64_t ended = __builtin_amdgcn_ballot_w64(any & (end <= first));
        if (ended == ~(uint64_t)0) continue;
        int at = __builtin_popcountll(ended);
#pragma unroll
        for (int r = 1; r < ROWS; ++r) {
            const int ended_by = __builtin_popcountll(__builtin_amdgcn_ballot_w64(any & (end <= first + r)));
            if (row >= first + r) at = ended_by;
        }
        b += at;
        if (ROWS > 1 && __builtin_amdgcn_ballot_w64(at == 64) != 0) {   // some row's sequence is not among these
            while (b < a.batch && a.cu[b + 1] <= row) ++b;
            return b < a.batch ? new_rows(a, b, max_rows) : NewRows{0, 0, 0, false};
        }
        const NewRows mine = {__shfl(s.first, at), __shfl(s.n, at), __shfl(s.start, at), __shfl(s.ok ? 1 : 0, at) != 0};
        return b < a.batch ? mine : NewRows{0, 0, 0, false};
    }
    return {0, 0, 0, false};
}

// Four e4m3 numbers times `scale`, a power of two, as bf16.
__device__ __forceinline__ u32x2 unpack_fp8(unsigned x, float scale) {
    return {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false)),
            __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true))};
}
// Eight e2m1 numbers times `scale`, a power of two (NaN where its exponent is 255), as bf16.
__device__ __forceinline__ u32x4 unpack_fp4(unsigned x, float scale) {
    return {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0)), __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1)),
            __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2)), __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3))};
}
__device__ __forceinline__ float power_of_two(int biased) { return __builtin_bit_cast(float, biased << 23); }

}  // namespace
#endif

#endif
