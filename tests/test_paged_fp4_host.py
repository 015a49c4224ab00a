"""The 4-bit paged cache without a GPU: refusals before any HIP call, and its definition against the bounds that it promises."""
import ctypes as C

import pytest
import torch

from tests.paged_fp4 import LEVELS, e2m1
from tests.test_paged_host import INVALID, PTR, TOO_SMALL, UNSUPPORTED, cache, fwd, move


def cache4(**more):
    return cache(**{**dict(format=2, k_exp=PTR, v_exp=PTR), **more})


@pytest.mark.parametrize("bad", [dict(k_exp=None), dict(v_exp=None), dict(k_exp=PTR + 2), dict(v_exp=PTR + 1), dict(format=3), dict(page_rows=12), dict(k=PTR + 8),
                                 dict(strides=(C.c_int64 * 3)(4096, 2048, 40)), dict(strides=(C.c_int64 * 3)(4096, 2048, 0))], ids=lambda x: "-".join(x))
def test_refusals(bad):
    c = cache4(**bad)
    assert move("ksa_paged_append", c=c) == INVALID and move("ksa_paged_read", c=c) == INVALID and fwd(c=c) == INVALID


def test_calls_that_are_fine_until_the_workspace_is_looked_at():
    assert fwd(c=cache4()) == TOO_SMALL
    assert fwd(c=cache4(strides=(C.c_int64 * 3)(4096, 2048, 64))) == TOO_SMALL
    assert move("ksa_paged_append", c=cache4(), total=0, k=None, v=None) == 0


def test_the_definition_rounds_to_the_nearest_and_loses_no_more_than_half_a_step():
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(500, 64, generator=g) * torch.exp2(20 * torch.randn(500, 1, generator=g))).to(torch.bfloat16).double()
    value, code, e = e2m1(x)
    scale = torch.exp2(e.double() - 127).repeat_interleave(32, -1)
    y = x / scale
    assert float(y.abs().max()) <= 7.0 and bool((y.abs().unflatten(-1, (-1, 32)).amax(-1) > 3.5).all())
    step = torch.where(y.abs() >= 4, 2.0, torch.where(y.abs() >= 2, 1.0, 0.5))
    assert bool(((value / scale - y).abs() <= step / 2).all())
    assert bool((LEVELS[(code % 8).long()] * scale == value.abs()).all())
    halfway = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0] + [0.0] * 24, dtype=torch.float64)
    assert e2m1(halfway)[0][:8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]


def test_pages_too_far_apart_are_refused():
    """Places within a page, and from page to page, are 32 bits."""
    for strides in ((2 ** 32, 2048, 64), (2 ** 40, 2048, 64), (2 ** 33, 2048, 2 ** 28), (4096, 2048, 2 ** 28)):
        c = cache4(strides=(C.c_int64 * 3)(*strides))
        assert move("ksa_paged_append", c=c) == UNSUPPORTED and move("ksa_paged_read", c=c) == UNSUPPORTED and fwd(c=c) == UNSUPPORTED, strides
    for strides in ((2 ** 32 - 16, 2048, 64), (2 ** 32 - 16, 2 ** 40, 64), (4096, 2048, 2 ** 28 - 16)):      # (16 rows; heads may lie anywhere)
        assert fwd(c=cache4(strides=(C.c_int64 * 3)(*strides))) == TOO_SMALL, strides
