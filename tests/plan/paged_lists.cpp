// Which listed keys no row of the group sees, on the host: none where the rows are of one kind, and of both kinds only summaries between those that the
// text rows see and those that the summary rows see.  Prints the most there were of these, or the first fault.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>

using std::max;
using std::min;
struct KsaDivisor {
    int d;
};
static int ksa_div(int x, const KsaDivisor &d) { return x / d.d; }
#include "ksa_paged_index.h"

static int unseen(const PagedRows &a, const Keys &k, int from, int to, int kinds, bool between) {
    int n = 0;
    for (int x = 0; x < k.n; ++x) {
        bool any = false;
        int text_end = 0, sums_begin = INT32_MAX;   // of the summaries that rows of either kind see
        for (int row = from; row <= to; ++row) {
            const RowKind r = kind_of(a, row);
            if (!((kinds >> (r.text ? 1 : 0)) & 1)) continue;
            const Visible v = visible(a, r);
            any |= seen_of(k, v).sees(x);
            if (r.text) text_end = max(text_end, v.hi_s);
            else sums_begin = min(sums_begin, v.lo_s);
        }
        if (any) continue;
        const RowKind key = key_at(k, x);
        if (!between || key.text || key.idx < text_end || key.idx >= sums_begin) {
            std::printf("fault: rows %d .. %d, c %d m %d C %d, key %d (%s %d) is seen by none\n", from, to, a.c, a.m, a.C, x, key.text ? "text" : "summary", key.idx);
            std::exit(1);
        }
        ++n;
    }
    return n;
}

int main() {
    const int shapes[][4] = {{4, 2, 1, 0}, {4, 2, 1, 1}, {5, 1, 0, 0}, {6, 3, 2, 0}, {1, 0, 7, 0}, {4, 0, 2, 0}, {3, 3, 0, 1}, {8, 1, 100, 0}, {4, 0, 0, 0}, {1, 1, 3, 0}};
    int most = 0;
    for (const auto &sh : shapes) {
        PagedRows a = {};
        a.c = sh[0], a.m = sh[1], a.C = sh[2], a.self_only = sh[3];
        a.by_w = {a.c + a.m}, a.by_c = {a.c}, a.by_m = {max(a.m, 1)};
        const int L = 41 / a.c * (a.c + a.m) + 41 % a.c;
        for (int from = 0; from < L; ++from)
            for (int to = from; to < min(from + 14, L); ++to) {
                const int of_all = unseen(a, keys_of(a, from, to), from, to, 3, true);
                if (of_all > a.C * a.m) {
                    std::printf("fault: %d listed keys that no row sees, rows %d .. %d\n", of_all, from, to);
                    return 1;
                }
                most = max(most, of_all);
                for (int kind = 0; kind < 2; ++kind) {   // the first and the last row of a kind
                    int first = -1, last = -1;
                    for (int row = from; row <= to; ++row)
                        if (kind_of(a, row).text == (kind == 1)) last = row, first = first < 0 ? row : first;
                    if (first >= 0) unseen(a, keys_between(visible(a, kind_of(a, first)), visible(a, kind_of(a, last))), from, to, 1 << kind, false);
                }
            }
    }
    std::printf("%d\n", most);
    return 0;
}
