"""GPU tests of 8-bit caches whose exponent bytes are outside the format (a slot never written holds any byte): they reach no row that does not
see theirs."""
import numpy as np
import pytest
import torch

import paper_2604_24432_amd as K
from tests.paged import Pages, batch_of, kinds, mask, randn

pytestmark = pytest.mark.gpu

WILD = [(247, 0x7e), (250, 0xfe), (254, 0x01), (255, 0x7e), (255, 0x00), (0, 0x7e)]     # exponent, payload (none of them NaN)


def bits(t):
    return t.contiguous().view(torch.int16)


def spoil(pages, rows, heads, exponent, byte, of):
    """Rows `rows` of sequence 0 become `byte` times 2^(exponent - 127) in the K or V pool, past the library."""
    pool, exp = (pages.k, pages.k_exp) if of == "k" else (pages.v, pages.v_exp)
    _, text, idx = kinds(int(rows.max()) + 1, pages.p.chunk_len, pages.p.n_summary)
    for row in rows:
        table = pages.text if text[row] else pages.sums
        at, slot = int(table[0, idx[row] // pages.page]), int(idx[row] % pages.page)
        pool.view(torch.uint8)[at, heads, slot] = byte
        exp[at, heads, slot] = exponent


# c, m, C, heads, KV heads, d, text rows of the chunk, text rows of the next one: with the chunk's summaries between them
HOLES = [(16, 2, 2, 2, 1, 64, 2, 0), (16, 2, 2, 4, 2, 128, 1, 1), (8, 1, 30, 4, 1, 128, 3, 1), (64, 8, 1, 3, 1, 64, 2, 0), (8, 1, 30, 2, 1, 64, 1, 2)]


@pytest.mark.parametrize("n_splits", [1, 2, 9])
@pytest.mark.parametrize("case", HOLES, ids=lambda x: "x".join(map(str, x)))
def test_summaries_between_those_that_text_and_summary_rows_see(case, n_splits):
    """A call of text and summary rows lists the summaries between the two ranges, which no row sees: their pages may hold anything."""
    c, m, C, Hq, Hkv, d, before, after = case
    print(f"paged holes {case} splits={n_splits}", flush=True)
    w = c + m
    first, rows = 40 * w + c - before, before + m + after
    n = first + rows
    p = K.make_params(1, 4096, c, m, C, Hq, Hkv, d)
    assert rows * Hq // Hkv <= 32
    see = mask(np.arange(first, n), n, c, m, C)
    _, text, idx = kinds(n, c, m)
    hole = np.nonzero(~text & ~see.any(0) & (idx < idx[~text & see.any(0)].max()))[0]
    assert len(hole) >= m
    pages = Pages(p, [n], 8, True, 5)
    pages.put(0, 0, randn(n, Hkv, d, seed=6), randn(n, Hkv, d, seed=7))
    q = randn(rows, Hq, d, seed=8)
    cu, start = batch_of([first], [rows])
    o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=n_splits)
    assert bool(torch.isfinite(o0.float()).all()) and bool(torch.isfinite(lse0).all())
    for exponent, byte in WILD:
        for of in ("k", "v"):
            spoil(pages, hole, slice(None), exponent, byte, of)
        o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=n_splits)
        assert torch.equal(bits(o), bits(o0)) and torch.equal(lse, lse0), (exponent, byte)


# heads, KV heads, d, text tokens to reckon with, new rows, spans: few rows, tiles of 128 pairs, of 128 whose keys two groups of waves share, of 256
TILES = [(4, 2, 64, 4096, 9, 1), (4, 2, 128, 4096, 9, 2), (16, 2, 64, 2048, 65, 1), (16, 2, 128, 2048, 300, 3), (4, 2, 64, 16384, 300, 1),
         (4, 2, 128, 16384, 300, 1), (64, 2, 64, 16384, 1100, 1), (64, 2, 128, 16384, 1100, 1)]


@pytest.mark.parametrize("case", TILES, ids=lambda x: "x".join(map(str, x)))
def test_rows_that_do_not_see_a_row_of_any_exponent(case):
    Hq, Hkv, d, n_text, rows, n_splits = case
    print(f"paged wild exponents {case}", flush=True)
    p = K.make_params(1, n_text, 16, 2, 2, Hq, Hkv, d)
    first = 1233
    n, G = first + rows, Hq // Hkv
    see = mask(np.arange(first, n), n, 16, 2, 2)
    pages = Pages(p, [n], 8, True, 5)
    k, v = randn(n, Hkv, d, seed=6), randn(n, Hkv, d, seed=7)
    q = randn(rows, Hq, d, seed=8)
    cu, start = batch_of([first], [rows])
    pages.put(0, 0, k, v)
    o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=n_splits)
    assert bool(torch.isfinite(o0.float()).all())
    for at in (n - 1, n - 1 - rows // 2, n - rows // 3, first - 3):
        sees = torch.from_numpy(see[:, at]).cuda()
        for exponent, byte in WILD:
            for of in ("k", "v"):
                spoil(pages, np.array([at]), 0, exponent, byte, of)
                o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=n_splits)
                assert torch.equal(bits(o[~sees]), bits(o0[~sees])) and torch.equal(lse[~sees], lse0[~sees]), (at, exponent, byte, of)
                assert torch.equal(bits(o[:, G:]), bits(o0[:, G:])) and torch.equal(lse[:, G:], lse0[:, G:])     # the other KV heads'
                pages.put(0, 0, k, v)
