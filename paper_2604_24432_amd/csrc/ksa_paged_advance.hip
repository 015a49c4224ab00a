// A step's rows and pages from the sequences' lengths.  Integer work, bound by the latency of launches and of loads one behind the other; what is read are the
// tables' columns, once, and the reference counts, once.  Three kernels, each of which needs all of the one before it: every sequence gives back what it
// does not need and counts its rows and the columns that lack a page; the free pages become a map of bits; every sequence adds up what those before it
// want, takes the free pages of these ranks and describes its rows.  Many rows have a kernel of their own.  No
// result depends on the order of atomics: they count references down and nothing reads them in between.  64 sequences of 2300 columns, one token each,
// 13000 pages 4.1, 2.1 and 6.3 us; 200 sequences, 278000 rows, 12000 pages taken of 24000 4.8, 3.0, 9.0 and 5.4.  As five kernels, with sums and a list of the free pages of their own,
// 22 and 27 us for both; with the list written bit by bit by a thread per run of words the third kernel took 18.
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
    int32_t *want, *count, *text; // [batch]: columns that lack a page, rows, text rows
    int32_t *want_before, *text_before;   // [batch + 1]: what those of the sequences before add up to
    uint64_t *free_bits;          // [n_pages / 64]
    int32_t words;                // of free_bits
    bool rows_here;               // the sequences' own workgroups describe their rows
};

// Threads of a workgroup; pages of one that looks for free ones.
constexpr int N = 256, PAGES = 1024;
// Up to here every workgroup adds up all sequences' counts itself, above one workgroup does it for all, beside those that look for free pages. Each itself and one for all (us):
// 300 sequences 14.4 and 16.1, 2000 23.0 and 30.2, 4000 40 and 54, 16000 214 and 187.
constexpr int SUMS_EACH = 4096;
// Up to so many rows the sequences' own workgroups describe them, above a launch more does.  The host knows how long the maps are, and not how many of their rows are one
// sequence's, which takes 256 of them at a time.  Own workgroups and a launch more (us): 64 rows of 64 sequences 10.7 and 13.3, 7720 of 256 12.1 and 16.0; 56 single rows beside eight
// times 250 12.4 and 15.3, 500 13.1 and 15.4, 1000 14.3 and 16.1; but 63 beside one of 1000 13.2 and 14.9, 2000 14.8 and 15.1, 4000 17.8 and 15.0, 7500 23.2 and 14.8, so that
// from 2000 rows of one sequence on the line is too high by up to 8 us.
constexpr int ROWS_EACH = 8192;

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

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
// Sums of K numbers over a workgroup, in all threads.
template <int K>
__device__ __forceinline__ void block_sums(int64_t (&x)[K], int64_t (*shared)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = wave_sum(x[k]);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) shared[threadIdx.x >> 6][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        x[k] = 0;
#pragma unroll
        for (int w = 0; w < N / 64; ++w) x[k] += shared[w][k];
    }
    __syncthreads();
}
// Of the threads before this one; `all`: of all.
template <class T>
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

// Entries of a table's row, `step` apart, several on their way at once.
template <class F>
__device__ __forceinline__ void each_entry(const int32_t *row, int from, int to, F &&f) {
    constexpr int AT_ONCE = 8;
    for (int x0 = from + threadIdx.x; x0 < to; x0 += N * AT_ONCE) {
        int entry[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) entry[i] = row[min(x0 + i * N, to - 1)];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            if (x0 + i * N < to) f(x0 + i * N, entry[i]);
    }
}

__global__ __launch_bounds__(N) void ksa_advance_count_kernel(const Args a) {
    __shared__ int64_t shared[N / 64][1];
    const int b = blockIdx.x;
    const Step s = step_of(a, b);
    int32_t *const text = a.text_table + (int64_t)b * a.rows.text_cols, *const sums = a.sum_table + (int64_t)b * a.rows.sum_cols;
    int64_t lacks[1] = {0};
    if (s.ok) {
        auto give_back = [&](int32_t *row) {
            return [&a, row](int x, int page) {
                if (!names_page(a, page)) return;
                atomicSub(a.refs + page, 1);
                row[x] = -1;
            };
        };
        each_entry(text, 0, s.ended ? a.rows.text_cols : s.begin, give_back(text));
        if (s.ended) each_entry(sums, 0, a.rows.sum_cols, give_back(sums));
        each_entry(text, s.t0, s.t1, [&](int, int page) { lacks[0] += !names_page(a, page); });
        each_entry(sums, s.s0, s.s1, [&](int, int page) { lacks[0] += !names_page(a, page); });
    }
    block_sums(lacks, shared);
    if (threadIdx.x == 0) a.want[b] = (int)lacks[0], a.count[b] = s.rows, a.text[b] = s.text, a.start[b] = s.start;
}

// The free pages as bits; of many sequences also what those before each of them want and have, by the last workgroup.
__device__ __forceinline__ int clamped(int64_t x) { return (int)min(x, (int64_t)INT32_MAX); }
__global__ __launch_bounds__(N) void ksa_advance_free_kernel(const Args a) {
    const int64_t first = (int64_t)blockIdx.x * PAGES + threadIdx.x;
    if ((int)blockIdx.x < (a.words + PAGES / 64 - 1) / (PAGES / 64)) {
        int refs[PAGES / N];
#pragma unroll
        for (int x = 0; x < PAGES / N; ++x) refs[x] = a.refs[min(first + x * N, (int64_t)a.rows.n_pages - 1)];
#pragma unroll
        for (int x = 0; x < PAGES / N; ++x) {
            const int64_t page = first + x * N;
            const uint64_t bits = __builtin_amdgcn_ballot_w64(page < a.rows.n_pages && refs[x] == 0);
            if ((threadIdx.x & 63) == 0 && page < a.rows.n_pages) a.free_bits[page / 64] = bits;
        }
        return;
    }
    __shared__ int64_t shared[N / 64];
    int64_t before[3] = {0, 0, 0};
    const int32_t *const from[3] = {a.count, a.want, a.text};
    int32_t *const to[3] = {a.cu, a.want_before, a.text_before};
    for (int b0 = 0; b0 <= a.rows.batch; b0 += N) {
        const int b = b0 + threadIdx.x;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            int64_t all;
            const int64_t mine = before[k] + block_before<int64_t>(b < a.rows.batch ? from[k][b] : 0, shared, all);
            if (b <= a.rows.batch) to[k][b] = clamped(mine);
            before[k] += all;
        }
    }
}

__device__ __forceinline__ void describe(const Args &a, int row, int aug, int b, int text_before, int held) {
    const int j = ksa_div(aug, a.rows.by_w), in = aug - j * (a.rows.c + a.rows.m);
    const RowKind kind = kind_of(a.rows, aug);
    const Spot spot = spot_of(a.rows, entry_of(a.rows, b, kind));
    if (a.slots) a.slots[row] = spot.page >= 0 ? ((int64_t)spot.page << a.rows.shift) + spot.slot : -1;
    if (a.positions) a.positions[row] = j * a.rows.c + min(in, a.rows.c - 1);
    if (a.tokens) a.tokens[row] = kind.text ? clamped((int64_t)text_before + (kind.idx - held)) : -1 - (in - a.rows.c);
}
__device__ __forceinline__ void describe_none(const Args &a, int row) {
    if (a.slots) a.slots[row] = -1;
    if (a.positions) a.positions[row] = 0;
    if (a.tokens) a.tokens[row] = -1;
}

__global__ __launch_bounds__(N) void ksa_advance_take_kernel(const Args a) {
    __shared__ int64_t shared[N / 64][5];
    __shared__ int shared_int[N / 64], run_before[N];
    const int b = blockIdx.x, batch = a.rows.batch;
    // free pages in the thread's run of words, and in those before it
    const int each = (a.words + N - 1) / N, w0 = min((int)threadIdx.x * each, a.words), w1 = min(w0 + each, a.words);
    int free_here = 0, n_free;
    for (int w = w0; w < w1; ++w) free_here += __builtin_popcountll(a.free_bits[w]);
    const int want = a.want[b];
    const Step s = step_of(a, b);
    // rows and text of the sequences before, rows and wants of all
    int rows_before, want_before, text_before, all_rows, all_want;
    if (batch <= SUMS_EACH) {
        int64_t x[5] = {0, 0, 0, 0, 0};
        for (int y = threadIdx.x; y < batch; y += N) {
            const int rows = a.count[y], want = a.want[y], text = a.text[y];
            if (y < b) x[0] += rows, x[1] += want, x[2] += text;
            x[3] += rows, x[4] += want;
        }
        block_sums(x, shared);
        rows_before = clamped(x[0]), want_before = clamped(x[1]), text_before = clamped(x[2]), all_rows = clamped(x[3]), all_want = clamped(x[4]);
        if (threadIdx.x == 0) {
            a.cu[b] = rows_before, a.text_before[b] = text_before;
            if (b == 0) a.cu[batch] = all_rows;
        }
    } else {
        rows_before = a.cu[b], want_before = a.want_before[b], text_before = a.text_before[b], all_rows = a.cu[batch], all_want = a.want_before[batch];
    }
    run_before[threadIdx.x] = block_before<int>(free_here, shared_int, n_free);
    __syncthreads();
    if (b == 0 && threadIdx.x == 0) *a.lacking = max(all_want - n_free, 0);
    const int end = min(want_before + want, n_free);
    if (end > want_before) {   // (the same in all threads)
        // the page of a rank: the run of words that holds it, the word, the bit
        auto page_of = [&](int rank) {
            int lo = 0, hi = N;
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (run_before[mid] <= rank) lo = mid;
                else hi = mid;
            }
            int left = rank - run_before[lo], w = lo * each;
            uint64_t bits = a.free_bits[w];
            for (int n = __builtin_popcountll(bits); left >= n; n = __builtin_popcountll(bits)) left -= n, bits = a.free_bits[++w];
            int at = 0;
#pragma unroll
            for (int half = 32; half > 0; half >>= 1) {
                const int n = __builtin_popcountll(bits >> at & ((1ull << half) - 1));
                if (left >= n) left -= n, at += half;
            }
            return w * 64 + at;
        };
        int at = want_before;
        auto take = [&](int32_t *table, int from, int to) {
            for (int x0 = from; x0 < to && at < end; x0 += N) {   // (the same in all threads)
                const int x = x0 + threadIdx.x, lacks = x < to && !names_page(a, table[x]);
                int all;
                const int mine = at + block_before<int>(lacks, shared_int, all);
                if (lacks && mine < end) {
                    const int page = page_of(mine);
                    table[x] = page, a.refs[page] = 1;
                }
                at += all;
            }
        };
        take(a.text_table + (int64_t)b * a.rows.text_cols, s.t0, s.t1);
        take(a.sum_table + (int64_t)b * a.rows.sum_cols, s.s0, s.s1);
        __syncthreads();
    }
    if (!a.rows_here) return;
    const int held = a.held[b], mapped = min(s.rows, a.rows.total - rows_before);   // (a row's place may be beyond 32 bits where it is beyond the maps)
    for (int x = threadIdx.x; x < mapped; x += N) describe(a, rows_before + x, s.start + x, b, text_before, held);
    for (int64_t row = (int64_t)all_rows + b * N + threadIdx.x; row < a.rows.total; row += (int64_t)batch * N) describe_none(a, (int)row);
}

__global__ __launch_bounds__(N) void ksa_advance_rows_kernel(const Args a) {
    const int row = blockIdx.x * N + threadIdx.x;
    if (row >= a.rows.total) return;
    if (row >= a.cu[a.rows.batch]) return describe_none(a, row);
    int lo = 0, hi = a.rows.batch;   // the last sequence that begins at or in front of the row
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.cu[mid] <= row) lo = mid;
        else hi = mid;
    }
    describe(a, row, a.start[lo] + (row - a.cu[lo]), lo, a.text_before[lo], a.held[lo]);
}

}  // namespace

size_t ksa_paged_advance_ints(int32_t batch, int32_t n_pages) { return 5 * (size_t)batch + 2 + 2 * (((size_t)n_pages + 63) / 64); }

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
    a.words = (int)(((int64_t)a.rows.n_pages + 63) / 64);
    int32_t *w = L.workspace;
    auto room = [&](int64_t n) {
        int32_t *const at = w;
        w += n;
        return at;
    };
    a.free_bits = reinterpret_cast<uint64_t *>(room(2 * (int64_t)a.words));   // (first: on 8 bytes)
    a.want = room(batch), a.count = room(batch), a.text = room(batch), a.want_before = room(batch + 1), a.text_before = room(batch + 1);
    const bool maps = a.rows.total > 0 && (a.slots || a.positions || a.tokens);
    a.rows_here = maps && a.rows.total <= ROWS_EACH;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int blocks = (a.words + PAGES / 64 - 1) / (PAGES / 64);
    hipLaunchKernelGGL(ksa_advance_count_kernel, dim3(batch), dim3(N), 0, st, a);
    hipLaunchKernelGGL(ksa_advance_free_kernel, dim3(batch > SUMS_EACH ? blocks + 1 : blocks), dim3(N), 0, st, a);
    hipLaunchKernelGGL(ksa_advance_take_kernel, dim3(batch), dim3(N), 0, st, a);
    if (maps && !a.rows_here) hipLaunchKernelGGL(ksa_advance_rows_kernel, dim3((unsigned)(((int64_t)a.rows.total + N - 1) / N)), dim3(N), 0, st, a);
    return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
}
