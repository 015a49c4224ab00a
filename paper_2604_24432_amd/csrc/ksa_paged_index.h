// Which rows a call's new rows see and where they lie: the integer side of the paged cache's kernels.  No HIP in here, so that it also
// compiles for the host, where every index is checked against the definitions.  Needs KsaDivisor and ksa_div.
#ifndef KSA_PAGED_INDEX_H_
#define KSA_PAGED_INDEX_H_

#ifdef __HIPCC__
#define KSA_INDEX __device__ __forceinline__
#else
#define KSA_INDEX inline
#endif

namespace {

struct PagedRows {
    const int32_t *text_table, *sum_table;
    int32_t text_cols, sum_cols, n_pages, shift;
    const int32_t *cu, *start;
    int32_t batch, total, aug_len;
    int32_t c, m, C, self_only;
    KsaDivisor by_w, by_c, by_m;          // c + m, c, m
};

// A sequence's new rows: packed rows first .. first + n - 1 are augmented rows start, start + 1, ...; !ok: out of place.
struct NewRows {
    int first, n, start;
    bool ok;
};
KSA_INDEX NewRows new_rows(const PagedRows &a, int b, int max_rows) {
    const int c0 = a.cu[b], c1 = a.cu[b + 1], at = a.start[b];
    const int lo = min(max(c0, 0), a.total), hi = min(max(c1, 0), a.total);
    NewRows r = {lo, max(hi - lo, 0), at, true};
    r.ok = lo == c0 && hi == c1 && r.n <= max_rows && at >= 0 && r.n <= a.aug_len && at <= a.aug_len - r.n;
    return r;
}

// An augmented row's kind, and its text index or summary ordinal (Eq. 1).
struct RowKind {
    bool text;
    int idx;
};
KSA_INDEX RowKind kind_of(const PagedRows &a, int row) {
    const int j = ksa_div(row, a.by_w), in = row - j * (a.c + a.m);
    return {in < a.c, in < a.c ? j * a.c + in : j * a.m + in - a.c};
}
KSA_INDEX int row_of(const PagedRows &a, RowKind k) {
    return k.text ? k.idx + ksa_div(k.idx, a.by_c) * a.m : k.idx + (ksa_div(k.idx, a.by_m) + 1) * a.c;
}
KSA_INDEX int text_before(const PagedRows &a, int row) {   // text rows among the first `row` augmented rows
    const int j = ksa_div(row, a.by_w);
    return j * a.c + min(row - j * (a.c + a.m), a.c);
}

// Where a row of one of the tables lies, in two steps, so that the first one's load may be on its way for a while.  entry_of: what the table
// says (its last column stands in for one behind it).  spot_of: page < 0 for no page.
struct Entry {
    int page, slot;
    bool inside;
};
struct Spot {
    int page, slot;
};
KSA_INDEX Entry entry_of(const PagedRows &a, int b, RowKind k) {
    // (values first: a choice between members of `a` is one between their addresses, and so a load from memory)
    const int32_t *const of_text = a.text_table, *const of_sums = a.sum_table, *const table = k.text ? of_text : of_sums;
    const int text_cols = a.text_cols, sum_cols = a.sum_cols, cols = k.text ? text_cols : sum_cols;
    const int col = k.idx >> a.shift;
    return {table[(int64_t)b * cols + min(col, cols - 1)], k.idx & ((1 << a.shift) - 1), col < cols};
}
KSA_INDEX Spot spot_of(const PagedRows &a, const Entry &e) { return {(e.inside & ((unsigned)e.page < (unsigned)a.n_pages)) ? e.page : -1, e.slot}; }

// What a row sees (Eq. 3): summaries [lo_s, hi_s), text [lo_t, hi_t).
struct Visible {
    int lo_s, hi_s, lo_t, hi_t;
};
KSA_INDEX Visible visible(const PagedRows &a, RowKind k) {
    if (k.text) {
        const int first = max(ksa_div(k.idx, a.by_c) - a.C, 0);
        return {0, first * a.m, first * a.c, k.idx + 1};
    }
    const int j = ksa_div(k.idx, a.by_m);
    return {a.self_only ? k.idx : j * a.m, k.idx + 1, j * a.c, (j + 1) * a.c};
}

// The list of keys that a group of rows sees together: positions [0, n_s) are summaries from s0 on, [n_s, n) text from t0 on.
struct Keys {
    int s0, n_s, t0, n;
};
KSA_INDEX RowKind key_at(const Keys &k, int x) { return {x >= k.n_s, x >= k.n_s ? k.t0 + (x - k.n_s) : k.s0 + x}; }
// ... of rows of one kind (ranges do not decrease from row to row)
KSA_INDEX Keys keys_between(const Visible &first, const Visible &last) {
    const int n_s = max(last.hi_s - first.lo_s, 0);
    return {first.lo_s, n_s, first.lo_t, n_s + last.hi_t - first.lo_t};
}
// ... of the augmented rows from .. to (both included).  Summaries between those that the text rows see and those that the summary rows see, up to C m,
// are listed too, though no row sees them.
KSA_INDEX Keys keys_of(const PagedRows &a, int from, int to) {
    const int c = a.c, m = a.m, w = c + m;
    const int j0 = ksa_div(from, a.by_w), r0 = from - j0 * w, j1 = ksa_div(to, a.by_w), r1 = to - j1 * w;
    int s_lo = INT32_MAX, s_hi = 0, t_lo = INT32_MAX, t_hi = 0;
    if (r0 < c || j1 > j0) {         // text rows
        const Visible first = visible(a, RowKind{true, r0 < c ? j0 * c + r0 : (j0 + 1) * c}), last = visible(a, RowKind{true, j1 * c + min(r1, c - 1)});
        t_lo = first.lo_t, t_hi = last.hi_t;
        if (last.hi_s > 0) s_lo = 0, s_hi = last.hi_s;
    }
    if (m > 0 && (r1 >= c || j1 > j0)) {   // summary rows
        const Visible first = visible(a, RowKind{false, j0 * m + max(r0 - c, 0)}), last = visible(a, RowKind{false, j1 * m - 1 + max(r1 - c + 1, 0)});
        s_lo = min(s_lo, first.lo_s), s_hi = max(s_hi, last.hi_s), t_lo = min(t_lo, first.lo_t), t_hi = max(t_hi, last.hi_t);
    }
    const int s0 = min(s_lo, s_hi);
    return {s0, s_hi - s0, t_lo, s_hi - s0 + t_hi - t_lo};
}

// A row's keys as positions of the list: [a, b) and [c, d), joined to one where they meet.
struct Seen {
    int a, b, c, d;
    // (no && and ||: they would become branches)
    KSA_INDEX bool sees(int x) const { return ((x >= a) & (x < b)) | ((x >= c) & (x < d)); }
    KSA_INDEX unsigned sees_32(int x) const {   // bit i: key x + i
        return (upto(b - x) & ~upto(a - x)) | (upto(d - x) & ~upto(c - x));
    }
    KSA_INDEX static unsigned upto(int n) { return n >= 32 ? ~0u : (1u << max(n, 0)) - 1; }   // the first n bits
    KSA_INDEX bool sees_all(int x, int end) const { return ((x >= a) & (end <= b)) | ((x >= c) & (end <= d)); }
    KSA_INDEX bool sees_any(int x, int end) const { return (max(x, a) < min(end, b)) | (max(x, c) < min(end, d)); }
};
KSA_INDEX Seen seen_of(const Keys &k, const Visible &v) {
    Seen s = {v.lo_s - k.s0, v.hi_s - k.s0, v.lo_t - k.t0 + k.n_s, v.hi_t - k.t0 + k.n_s};
    if (s.b <= s.a) s.a = s.b = s.c;   // no summaries
    if (s.b == s.c) s.b = s.c = s.d;
    return s;
}

}  // namespace

#endif
