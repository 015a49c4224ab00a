"""A step's rows and pages without a GPU: refusals before any HIP call, the workspace, and the tests' own model of it against what it promises."""
import ctypes as C
import random

import pytest

from paper_2604_24432_amd import binding
from tests.advance import advance
from tests.test_paged_host import INVALID, PTR, TOO_SMALL, UNSUPPORTED, cache, params

NAMES = ("page_refs", "held", "new_text", "cu_rows", "start", "lacking", "slots", "positions", "tokens")


def call(p=None, c=None, total=10, ws=PTR, ws_bytes=1 << 20, **ptr):
    p = params() if p is None else p
    c = cache() if c is None else c
    args = [ptr.get(x, PTR) for x in NAMES]
    return binding.lib().ksa_paged_advance(C.byref(p), C.byref(c) if c else None, *args, total, ws, ws_bytes, None)


def need(p, c):
    return binding.lib().ksa_paged_advance_workspace_bytes(C.byref(p), C.byref(c))


def test_refusals():
    for x in NAMES:
        if x not in ("slots", "positions", "tokens"):
            assert call(**{x: None}) == INVALID, x
        assert call(**{x: PTR + 2}) == INVALID, x
    assert call(slots=PTR + 4) == INVALID
    for bad in (dict(c=False), dict(total=-1), dict(ws=None), dict(ws=PTR + 8), dict(c=cache(page_rows=12)), dict(c=cache(n_pages=0)), dict(p=params(batch=0))):
        assert call(**bad) == INVALID, bad
    assert call(p=params(head_dim=32)) == UNSUPPORTED
    assert call(c=cache(text_pages=2 ** 30)) == UNSUPPORTED and need(params(), cache(text_pages=2 ** 30)) == 0
    assert call(total=2 ** 31) == UNSUPPORTED
    size = need(params(), cache())
    assert size > 0 and size % 16 == 0 and call(ws_bytes=size - 1) == TOO_SMALL


def test_the_workspace_grows_with_what_it_holds():
    sizes = [need(params(batch=b), cache(n_pages=n)) for b, n in ((1, 1), (2, 100), (300, 100), (300, 5000), (65535, 10 ** 7))]
    assert sizes == sorted(sizes) and sizes[-1] >= 10 ** 7 // 8 + 4 * 5 * 65535
    assert need(params(batch=0), cache()) == 0 and need(params(), cache(format=9)) == 0


@pytest.mark.parametrize("seed", range(20))
def test_the_model_keeps_its_books(seed):
    """Every page is named as often as it is counted, no two sequences have one, what new rows need is there, and a second call changes nothing."""
    g = random.Random(seed)
    c, m, C, page = g.choice([(8, 1, 2, 8), (16, 4, 0, 8), (12, 3, 1, 16), (1, 0, 30, 8), (64, 8, 1, 16)])
    n, B = 400, g.randint(1, 6)
    cols = -(-n // page), -(-(n // c * m) // page)
    text, sums = [[-1] * cols[0] for _ in range(B)], [[-1] * cols[1] for _ in range(B)]
    refs = [0] * g.choice([20, 60, 400])
    held, lost = [0] * B, [False] * B
    for _ in range(30):
        new = [g.choice([1, 1, 1, 0, g.randint(1, 90), -1]) for _ in range(B)]
        new = [min(t, n - h) for t, h in zip(new, held)]
        cu, start, lacking, rows = advance(c, m, C, page, n, text, sums, refs, held, new)
        count = [0] * len(refs)
        for table in (*text, *sums):
            for entry in table:
                if entry >= 0:
                    count[entry] += 1
        assert count == refs and max(refs) <= 1
        before = [list(map(list, text)), list(map(list, sums)), list(refs)]
        again = advance(c, m, C, page, n, text, sums, refs, held, new)
        assert again[0] == cu and again[3] == rows and [text, sums, refs] == before
        assert lacking > 0 or all(r[0] >= 0 for b in range(B) if not lost[b] for r in rows[cu[b]:cu[b + 1]])
        assert len({r[0] for r in rows if r[0] >= 0}) == sum(r[0] >= 0 for r in rows)
        for b in range(B):
            lost[b] = new[b] >= 0 and (lost[b] or any(r[0] < 0 for r in rows[cu[b]:cu[b + 1]]))
            held[b] = 0 if new[b] < 0 else held[b] + new[b]


def test_columns_and_rows_whose_steps_pass_32_bits_are_refused():
    """A workgroup goes over columns 2048 at a time: a step behind the last one has to fit 32 bits too."""
    p, c = params(batch=1), lambda n: cache(text_pages=n, summary_pages=8)
    for n in (2 ** 31 - 4096 - 8, 2 ** 31 - 2048, 2 ** 31 - 9, 2 ** 31 - 1):
        assert call(p=p, c=c(n)) == UNSUPPORTED and need(p, c(n)) == 0, n
    assert need(p, c(2 ** 31 - 4096 - 9)) > 0 and call(p=p, c=c(2 ** 31 - 4096 - 9), ws_bytes=0) == TOO_SMALL
    assert call(total=2 ** 31 - 256) == UNSUPPORTED and call(total=2 ** 31 - 257, ws_bytes=0) == TOO_SMALL
