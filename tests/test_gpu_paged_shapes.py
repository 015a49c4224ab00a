"""GPU tests of the paged cache at the ends of its parameters' ranges."""
import pytest
import torch

import paper_2604_24432_amd as K
from tests.paged import Pages, attend, batch_of, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("c,m", [(2 ** 31 - 1, 1), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 2, 2 ** 30 - 1), (10 ** 9, 10 ** 9), (101, 101)])
def test_chunks_longer_than_any_text(c, m, rows):
    """No chunk is ever whole: rows see all text up to themselves."""
    print(f"paged long chunks c={c} m={m} rows={rows}", flush=True)
    p = K.make_params(1, 100, c, m, 1, 4, 2, 64)
    pages = Pages(p, [100], 16, False, 5)
    k, v, q = randn(100, 2, 64, seed=1), randn(100, 2, 64, seed=2), randn(rows, 4, 64, seed=3)
    K.ksa_paged_append(pages.cache, k, v, *batch_of([0], [100]))
    k2, v2 = K.ksa_paged_read(pages.cache, *batch_of([0], [100]), 100)
    assert torch.equal(k2.view(torch.int16), k.view(torch.int16)) and torch.equal(v2.view(torch.int16), v.view(torch.int16))
    o, lse = K.ksa_paged_fwd(pages.cache, q, *batch_of([100 - rows], [rows]))
    plain = K.make_params(1, 100, 1, 0, 200, 4, 2, 64)     # the same rows and keys, as a window longer than the text
    want, want_lse, off, lse_off = attend(q.double(), k.double(), v.double(), list(range(100 - rows, 100)), plain)
    assert bool(((o.double() - want).abs() <= off).all()) and bool(((lse.double() - want_lse).abs() <= lse_off).all())


# heads, KV heads, d, text tokens to reckon with, rows of two sequences, spans: every kernel, every way of joining spans
CALLS = [(32, 8, 128, 8192, (1, 1), 0), (8, 1, 64, 8192, (3, 2), 5), (32, 8, 128, 8192, (2, 1), 2), (16, 2, 64, 2048, (65, 40), 1), (16, 2, 128, 2048, (300, 1), 3),
         (4, 2, 64, 16384, (300, 20), 1), (4, 2, 128, 16384, (300, 20), 9), (64, 2, 64, 16384, (1100, 900), 1), (64, 2, 128, 16384, (1100, 900), 4)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", CALLS, ids=str)
def test_the_same_call_gives_the_same_bits(case, fp8):
    Hq, Hkv, d, n_text, rows, n_splits = case
    print(f"paged repeated calls {case} fp8={fp8}", flush=True)
    p = K.make_params(2, n_text, 16, 2, 2, Hq, Hkv, d)
    L = [1700, 1233]
    pages = Pages(p, L, 16, fp8, 5)
    for b in range(2):
        pages.put(b, 0, randn(L[b], Hkv, d, seed=b), randn(L[b], Hkv, d, seed=b + 5))
    q = randn(sum(rows), Hq, d, seed=9)
    cu, start = batch_of([n - r for n, r in zip(L, rows)], rows)
    o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=max(rows), n_splits=n_splits)
    for turn in range(6):
        if turn % 2:      # something else on the chip meanwhile, in front of the call and beside it
            other = torch.cuda.Stream()
            with torch.cuda.stream(other):
                x = torch.randn(1024, 1024, device="cuda")
                for _ in range(4):
                    x = x @ x * 1e-3
        o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=max(rows), n_splits=n_splits)
        assert torch.equal(o.view(torch.int16), o0.view(torch.int16)) and torch.equal(lse, lse0)
        torch.cuda.synchronize()
