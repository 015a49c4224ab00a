// A step's rows and pages from the sequences' lengths.  Integer work, bound by the latency of launches and of loads one behind the other; what is read are the
// tables' columns, once, and the reference counts, once.  Five kernels, each of which needs all of the one before it: every sequence gives back what it
// does not need and counts its rows and the columns that lack a page; the counts are summed up, and so are the free pages, in blocks; the free pages
// that are wanted are listed in order; every sequence takes its own; rows are described.  No result depends on the order of atomics: they count
// references down and nothing reads them in between.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ksa_paged.h"

namespace {

struct Args {
    PagedRows rows;               // (cu and start: where they go)
    int32_t *text_table, *sum_table, *refs;
    const int32_t *held, *new_text;
    int32_t *cu, *start, *lacking;
    int64_t *slots;
    int32_t *positions, *tokens;
    int32_t n_text;
    int32_t *want, *count, *text; // [batch]: columns that lack a page, rows, text rows; then what those of the sequences before add up to (want, text: [batch + 1])
    int32_t *want_before, *text_before;
    int32_t *free_in, *free_all;  // [blocks of pages]: free pages; [1]
    int32_t *list;                // [n_pages]: free pages in order
    int32_t blocks;
};

constexpr int PAGES = 4096;       // of a block

// What a sequence does in a step (columns: of text, of summaries).
struct Step {
    bool ok, ended;
    int start, rows, text;
    int begin;                    // text columns before this one are given back
    int t0, t1, s0, s1;           // columns [t0, t1), [s0, s1) that begin with a new row or behind the first, and hold one
};
__device__ __forceinline__ Step step_of(const Args &a, int b) {
    const int h = a.held[b], t = a.new_text[b];
    Step s = {true, t < 0, 0, 0, 0, 0, 0, 0, 0, 0};
    if (s.ended) return s;
    if (h < 0 || h > a.n_text || t > a.n_text - h) {
        s.ok = false, s.start = -1;
        return s;
    }
    const PagedRows &r = a.rows;
    const int e = h + t, j = ksa_div(h, r.by_c), je = ksa_div(e, r.by_c), mask = (1 << r.shift) - 1;
    auto columns = [&](int n) { return (n >> r.shift) + ((n & mask) ? 1 : 0); };
    s.start = h + j * r.m, s.text = t, s.rows = t + (je - j) * r.m;
    s.begin = min((max(j - r.C, 0) * r.c) >> r.shift, r.text_cols);
    s.t0 = min(columns(h), r.text_cols), s.t1 = min(columns(e), r.text_cols);
    s.s0 = min(columns(j * r.m), r.sum_cols), s.s1 = min(columns(je * r.m), r.sum_cols);
    return s;
}
__device__ __forceinline__ bool names_page(const Args &a, int entry) { return (unsigned)entry < (unsigned)a.rows.n_pages; }

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
// The sum of x over a block of N threads, in all of them.
template <int N>
__device__ __forceinline__ int block_sum(int x, int *shared) {
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    int y = 0;
#pragma unroll
    for (int w = 0; w < N / 64; ++w) y += shared[w];
    __syncthreads();
    return y;
}
// Of the threads before this one; `all`: of all.
template <int N, class T>
__device__ __forceinline__ T block_before(T x, T *shared, T &all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T upto = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T y = __shfl_up(upto, d);
        upto += lane >= d ? y : 0;
    }
    if (lane == 63) shared[wave] = upto;
    __syncthreads();
    T before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < N / 64; ++w) {
        const T y = shared[w];
        before += w < wave ? y : 0, all += y;
    }
    __syncthreads();
    return before + upto - x;
}

__device__ __forceinline__ void give_back(const Args &a, int32_t *entry) {
    const int page = *entry;
    if (!names_page(a, page)) return;
    atomicSub(a.refs + page, 1);
    *entry = -1;
}

__global__ __launch_bounds__(256) void ksa_advance_count_kernel(const Args a) {
    __shared__ int shared[4];
    const int b = blockIdx.x;
    const Step s = step_of(a, b);
    int32_t *const text = a.text_table + (int64_t)b * a.rows.text_cols, *const sums = a.sum_table + (int64_t)b * a.rows.sum_cols;
    int lacks = 0;
    if (s.ok) {
        for (int x = threadIdx.x; x < (s.ended ? a.rows.text_cols : s.begin); x += 256) give_back(a, text + x);
        if (s.ended)
            for (int x = threadIdx.x; x < a.rows.sum_cols; x += 256) give_back(a, sums + x);
        for (int x = s.t0 + threadIdx.x; x < s.t1; x += 256) lacks += !names_page(a, text[x]);
        for (int x = s.s0 + threadIdx.x; x < s.s1; x += 256) lacks += !names_page(a, sums[x]);
    }
    lacks = block_sum<256>(lacks, shared);
    if (threadIdx.x == 0) a.want[b] = lacks, a.count[b] = s.rows, a.text[b] = s.text, a.start[b] = s.start;
}

// Block 0: sums over the sequences.  Block 1 + x: free pages of the x-th block of them.
__global__ __launch_bounds__(1024) void ksa_advance_sum_kernel(const Args a) {
    __shared__ int64_t shared[16];
    if (blockIdx.x > 0) {
        const int64_t first = (int64_t)(blockIdx.x - 1) * PAGES;
        int n = 0;
#pragma unroll
        for (int x = 0; x < PAGES / 1024; ++x) {
            const int64_t page = first + x * 1024 + threadIdx.x;
            n += page < a.rows.n_pages && a.refs[page] == 0;
        }
        n = block_sum<1024>(n, reinterpret_cast<int *>(shared));
        if (threadIdx.x == 0) a.free_in[blockIdx.x - 1] = n;
        return;
    }
    int64_t before[3] = {0, 0, 0};
    const int32_t *const from[3] = {a.count, a.want, a.text};
    int32_t *const to[3] = {a.cu, a.want_before, a.text_before};
    for (int b0 = 0; b0 <= a.rows.batch; b0 += 1024) {
        const int b = b0 + threadIdx.x;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            int64_t all;
            const int64_t mine = before[k] + block_before<1024, int64_t>(b < a.rows.batch ? from[k][b] : 0, shared, all);
            if (b <= a.rows.batch) to[k][b] = (int32_t)min(mine, (int64_t)INT32_MAX);
            before[k] += all;
        }
    }
}

// The free pages of a block of them, behind those of the blocks before, as far as they are wanted.
__global__ __launch_bounds__(1024) void ksa_advance_list_kernel(const Args a) {
    __shared__ int shared[16];
    int before = 0, all = 0;
    for (int x = threadIdx.x; x < a.blocks; x += 1024) {
        const int n = a.free_in[x];
        before += x < (int)blockIdx.x ? n : 0, all += n;
    }
    before = block_sum<1024>(before, shared);
    const int wanted = a.want_before[a.rows.batch];
    if (blockIdx.x == 0) {
        all = block_sum<1024>(all, shared);
        if (threadIdx.x == 0) *a.free_all = all, *a.lacking = max(wanted - all, 0);
    }
    if (before >= wanted) return;
    const int64_t first = (int64_t)blockIdx.x * PAGES + threadIdx.x * (PAGES / 1024);
    bool is_free[PAGES / 1024];
    int mine = 0;
#pragma unroll
    for (int x = 0; x < PAGES / 1024; ++x) is_free[x] = first + x < a.rows.n_pages && a.refs[first + x] == 0, mine += is_free[x];
    int in_block;
    int at = before + block_before<1024, int>(mine, shared, in_block);
#pragma unroll
    for (int x = 0; x < PAGES / 1024; ++x)
        if (is_free[x]) {
            if (at < wanted) a.list[at] = (int32_t)(first + x);
            ++at;
        }
}

__global__ __launch_bounds__(256) void ksa_advance_take_kernel(const Args a) {
    __shared__ int shared[4];
    const int b = blockIdx.x;
    const Step s = step_of(a, b);
    if (!s.ok || s.ended) return;
    int at = a.want_before[b];
    const int n_free = *a.free_all;
    auto take = [&](int32_t *table, int from, int to) {
        for (int x0 = from; x0 < to && at < n_free; x0 += 256) {   // (the same in all threads)
            const int x = x0 + threadIdx.x, lacks = x < to && !names_page(a, table[x]);
            int all;
            const int mine = at + block_before<256, int>(lacks, shared, all);
            if (lacks && mine < n_free) {
                const int page = a.list[mine];
                table[x] = page, a.refs[page] = 1;
            }
            at += all;
        }
    };
    take(a.text_table + (int64_t)b * a.rows.text_cols, s.t0, s.t1);
    take(a.sum_table + (int64_t)b * a.rows.sum_cols, s.s0, s.s1);
}

__global__ __launch_bounds__(256) void ksa_advance_rows_kernel(const Args a) {
    const int row = blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows.total) return;
    int64_t slot = -1;
    int position = 0, token = -1;
    if (row < a.cu[a.rows.batch]) {
        int lo = 0, hi = a.rows.batch;   // the last sequence that begins at or in front of the row
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.cu[mid] <= row) lo = mid;
            else hi = mid;
        }
        const int b = lo, aug = a.start[b] + (row - a.cu[b]), j = ksa_div(aug, a.rows.by_w), in = aug - j * (a.rows.c + a.rows.m);
        const RowKind kind = kind_of(a.rows, aug);
        const Spot spot = spot_of(a.rows, entry_of(a.rows, b, kind));
        if (spot.page >= 0) slot = ((int64_t)spot.page << a.rows.shift) + spot.slot;
        position = j * a.rows.c + min(in, a.rows.c - 1);
        token = kind.text ? (int)min((int64_t)a.text_before[b] + (kind.idx - a.held[b]), (int64_t)INT32_MAX) : -1 - (in - a.rows.c);
    }
    if (a.slots) a.slots[row] = slot;
    if (a.positions) a.positions[row] = position;
    if (a.tokens) a.tokens[row] = token;
}

}  // namespace

size_t ksa_paged_advance_ints(int32_t batch, int32_t n_pages) { return 5 * (size_t)batch + 2 + ((size_t)n_pages + PAGES - 1) / PAGES + 1 + (size_t)n_pages; }

int ksa_launch_paged_advance(const KsaPagedAdvance &L, void *stream) {
    Args a;
    a.rows = paged_rows(L.call);
    a.rows.cu = L.cu_rows, a.rows.start = L.start;
    a.text_table = const_cast<int32_t *>(L.call.cache.text_table), a.sum_table = const_cast<int32_t *>(L.call.cache.summary_table);
    a.refs = L.page_refs, a.held = L.held, a.new_text = L.new_text;
    a.cu = L.cu_rows, a.start = L.start, a.lacking = L.lacking;
    a.slots = L.slots, a.positions = L.positions, a.tokens = L.tokens;
    a.n_text = L.call.p.n_text;
    const int batch = a.rows.batch;
    a.blocks = (int)(((int64_t)a.rows.n_pages + PAGES - 1) / PAGES);
    int32_t *w = L.workspace;
    auto room = [&](int64_t n) {
        int32_t *const at = w;
        w += n;
        return at;
    };
    a.want = room(batch), a.count = room(batch), a.text = room(batch), a.want_before = room(batch + 1), a.text_before = room(batch + 1);
    a.free_in = room(a.blocks), a.free_all = room(1), a.list = room(a.rows.n_pages);
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(ksa_advance_count_kernel, dim3(batch), dim3(256), 0, st, a);
    hipLaunchKernelGGL(ksa_advance_sum_kernel, dim3(1 + a.blocks), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(ksa_advance_list_kernel, dim3(a.blocks), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(ksa_advance_take_kernel, dim3(batch), dim3(256), 0, st, a);
    if (a.rows.total > 0 && (a.slots || a.positions || a.tokens)) hipLaunchKernelGGL(ksa_advance_rows_kernel, dim3((a.rows.total + 255) / 256), dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
}
