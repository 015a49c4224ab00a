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
