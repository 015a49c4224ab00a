"""A step's rows and pages from the sequences' lengths, written out in Python, for the tests of the library's kernels."""


def advance(c, m, C, page, n_text, text, sums, refs, held, new):
    """Tables (lists of lists; changed), reference counts (changed), lengths -> cu_rows, start, lacking, rows as (slot, position, token)."""
    n_pages = len(refs)
    ok = lambda entry: 0 <= entry < n_pages  # noqa: E731
    aug = lambda n: n + n // c * m  # noqa: E731
    batch = len(held)
    state = []
    for b, (h, t) in enumerate(zip(held, new)):
        if t < 0:
            for table in (text, sums):
                for x, entry in enumerate(table[b]):
                    if ok(entry):
                        refs[entry] -= 1
                        table[b][x] = -1
            state.append("ended")
        elif h < 0 or h + t > n_text:
            state.append("out")
        else:
            first_seen = max(h // c - C, 0) * c             # by the next text row, and so by any later one
            for x, entry in enumerate(text[b]):
                if (x + 1) * page <= first_seen and ok(entry):
                    refs[entry] -= 1
                    text[b][x] = -1
            state.append("on")
    free = [x for x in range(n_pages) if refs[x] == 0]
    lacking, given = 0, 0
    for b, (h, t) in enumerate(zip(held, new)):
        if state[b] != "on":
            continue
        for table, lo, hi in ((text[b], h, h + t), (sums[b], h // c * m, (h + t) // c * m)):
            for x in range(len(table)):
                # the column's slots [x page, (x + 1) page) hold a new row, and none that was there before
                if x * page >= lo and x * page < hi and not ok(table[x]):
                    if given < len(free):
                        table[x] = free[given]
                        refs[free[given]] = 1
                        given += 1
                    else:
                        lacking += 1
    cu, start, rows, texts = [0], [], [], 0
    for b, (h, t) in enumerate(zip(held, new)):
        if state[b] != "on":
            start.append(-1 if state[b] == "out" else 0)
            cu.append(cu[-1])
            continue
        start.append(aug(h))
        for a in range(aug(h), aug(h + t)):
            j, r = divmod(a, c + m)
            table, idx = (text[b], j * c + r) if r < c else (sums[b], j * m + r - c)
            entry = table[idx // page] if idx // page < len(table) else -1
            rows.append((entry * page + idx % page if ok(entry) else -1, j * c + min(r, c - 1), texts + idx - h if r < c else c - 1 - r))
        texts += t
        cu.append(len(rows))
    return cu, start, lacking, rows
