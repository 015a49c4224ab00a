// Checks the index functions of the paged cache's kernels against the definitions, key by key, on the host: which keys a group of rows lists
// and sees (Eq. 3), which rows of a batch are in place, and that no table entry leads out of the pool.  Prints "ok" or the first fault.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

using std::max;
using std::min;
struct KsaDivisor {
    int d;
};
static int ksa_div(int x, const KsaDivisor &d) { return x / d.d; }
#include "ksa_paged_index.h"

static void fail(const char *what, int x, int y) {
    std::printf("fault: %s at %d, %d\n", what, x, y);
    std::exit(1);
}

static PagedRows rows_of(int c, int m, int C, int self_only) {
    PagedRows a = {};
    a.c = c, a.m = m, a.C = C, a.self_only = self_only;
    a.by_w = {c + m}, a.by_c = {c}, a.by_m = {m > 0 ? m : 1};
    return a;
}

// does augmented row x see augmented row y?
static bool sees(const PagedRows &a, int x, int y) {
    const int w = a.c + a.m, jx = x / w, jy = y / w;
    const bool tx = x % w < a.c, ty = y % w < a.c;
    if (tx) return ty ? jy >= jx - a.C && y <= x : jy < jx - a.C;
    return ty ? jy == jx : a.self_only ? x == y : jy == jx && y <= x;
}

static void check_list(const PagedRows &a, const Keys &k, const std::vector<int> &group, int L) {
    if (k.n_s < 0 || k.n <= k.n_s || k.s0 < 0 || k.t0 < 0) fail("list", k.n_s, k.n);
    std::vector<int> place(L, -1);   // list position of an augmented row
    for (int x = 0; x < k.n; ++x) {
        const RowKind r = key_at(k, x);
        const int row = row_of(a, r);
        if (row < 0 || row >= L) fail("row outside the sequence", row, L);
        const RowKind back = kind_of(a, row);
        if (back.text != r.text || back.idx != r.idx || place[row] != -1) fail("row listed twice", row, x);
        place[row] = x;
    }
    Seen every = {};
    for (const int q : group) {
        const Seen s = seen_of(k, visible(a, kind_of(a, q)));
        for (int y = 0; y < L; ++y) {
            if (sees(a, q, y) && place[y] < 0) fail("key not listed", q, y);
            if (place[y] >= 0 && s.sees(place[y]) != sees(a, q, y)) fail("key seen wrongly", q, y);
        }
        for (int x = 0; x < k.n; x += 8) {
            bool all = true, any = false;
            for (int y = x; y < x + 8; ++y) all &= s.sees(y), any |= s.sees(y);
            if (s.sees_all(x, x + 8) && !all) fail("not all are seen", q, x);
            if (s.sees_any(x, x + 8) != any) fail("any seen", q, x);
        }
        for (int x = -40; x < k.n + 40; x += 13)
            for (int i = 0; i < 32; ++i)
                if (((s.sees_32(x) >> i) & 1) != (s.sees(x + i) ? 1u : 0u)) fail("32 keys together", q, x);
        if (s.sees(-1) || s.sees(k.n)) fail("positions outside the list", q, k.n);
    }
    (void)every;
}

int main() {
    const int shapes[][4] = {{4, 2, 1, 0}, {4, 2, 1, 1}, {5, 1, 0, 0}, {6, 3, 2, 0}, {1, 0, 7, 0}, {4, 0, 2, 0}, {3, 3, 0, 1}, {8, 1, 100, 0}, {4, 0, 0, 0}, {1, 1, 3, 0}};
    for (const auto &sh : shapes) {
        PagedRows a = rows_of(sh[0], sh[1], sh[2], sh[3]);
        for (const int n_text : {41, 40, 12, 3}) {
            const int L = n_text / a.c * (a.c + a.m) + n_text % a.c;
            a.aug_len = L;
            int text = 0;
            for (int row = 0; row < L; ++row) {
                if (text_before(a, row) != text) fail("text in front of a row", row, text);
                text += kind_of(a, row).text;
            }
            for (int from = 0; from < L; ++from)
                for (int n = 1; n <= 12 && from + n <= L; ++n) {
                    std::vector<int> group, kinds[2];
                    for (int x = from; x < from + n; ++x) group.push_back(x), kinds[kind_of(a, x).text].push_back(x);
                    check_list(a, keys_of(a, from, from + n - 1), group, L);
                    for (const auto &g : kinds) {
                        if (g.empty()) continue;
                        const Visible lo = visible(a, kind_of(a, g.front())), hi = visible(a, kind_of(a, g.back()));
                        const Keys k = keys_between(lo, hi);
                        check_list(a, k, g, L);
                        const Seen every = seen_of(k, Visible{hi.lo_s, lo.hi_s, hi.lo_t, lo.hi_t});
                        for (int x = 0; x < k.n; ++x)
                            for (int len = 1; len <= 8; ++len)
                                if (every.sees_all(x, x + len))
                                    for (const int q : g)
                                        for (int y = x; y < x + len; ++y)
                                            if (!seen_of(k, visible(a, kind_of(a, q))).sees(y)) fail("not seen by every row", q, y);
                    }
                }
        }
    }
    // tables: an entry outside the pool and a column behind the table are no page
    PagedRows a = rows_of(4, 2, 1, 0);
    const int32_t text[2][3] = {{0, 4, -1}, {5, INT32_MIN, INT32_MAX}}, sums[2][1] = {{3}, {-7}};
    a.text_table = text[0], a.sum_table = sums[0], a.text_cols = 3, a.sum_cols = 1, a.n_pages = 5, a.shift = 3, a.batch = 2;
    for (int b = 0; b < 2; ++b)
        for (int idx : {0, 7, 8, 15, 16, 23, 24, 31, 1000, INT32_MAX})
            for (int kind = 0; kind < 2; ++kind) {
                const Spot s = spot_of(a, entry_of(a, b, RowKind{kind == 1, idx}));
                const int col = idx / 8, cols = kind ? 3 : 1, entry = col < cols ? (kind ? text[b][col] : sums[b][col]) : -1;
                const int want = entry >= 0 && entry < 5 ? entry : -1;
                if (s.page != want || s.slot != idx % 8) fail("page", b, idx);
            }
    // batches: what is in place, and no packed row outside the tensors whatever cu_rows holds
    const int32_t wild[] = {INT32_MIN, -1, 0, 3, 9, 10, 11, INT32_MAX};
    a.total = 10, a.aug_len = 20, a.batch = 1;
    for (const int32_t c0 : wild)
        for (const int32_t c1 : wild)
            for (const int32_t st : {INT32_MIN, -1, 0, 10, 17, 20, 21, INT32_MAX})
                for (const int most : {1, 7, 10}) {
                    const int32_t cu[2] = {c0, c1}, start[1] = {st};
                    a.cu = cu, a.start = start;
                    const NewRows r = new_rows(a, 0, most);
                    if (r.n < 0 || r.first < 0 || (int64_t)r.first + r.n > a.total) fail("packed rows", c0, c1);
                    const bool inside = c0 >= 0 && c0 <= 10 && c1 >= 0 && c1 <= 10;
                    const int64_t n = c1 > c0 ? (int64_t)c1 - c0 : 0;
                    if (inside && r.n != n) fail("number of rows", c0, c1);
                    if (r.ok != (inside && n <= most && st >= 0 && st + n <= 20)) fail("in place", c0, st);
                }
    std::printf("ok\n");
    return 0;
}
