"""GPU tests of the paged attention with a workspace that is not the one the library asks for."""
import pytest
import torch

import paper_2604_24432_amd as K
from tests.paged import Pages, attend, batch_of, randn, stands_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
def test_one_workspace_for_calls_of_any_size(fp8):
    """A loop that keeps one buffer: calls that would take more of it take fewer spans, with outputs of the same meaning."""
    print(f"paged workspaces fp8={fp8}", flush=True)
    p = K.make_params(2, 32768, 16, 2, 8, 8, 2, 128)
    L = [5000, 3111]
    pages = Pages(p, L, 16, fp8, 5)
    k, v = [randn(n, 2, 128, seed=b) for b, n in enumerate(L)], [randn(n, 2, 128, seed=5 + b) for b, n in enumerate(L)]
    for b in range(2):
        pages.put(b, 0, k[b], v[b])
    buffer = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    fewer = 0
    for rows in (1, 4, 60, 700):
        q = randn(2 * rows, 8, 128, seed=9)
        first = [n - rows for n in L]
        cu, start = batch_of(first, [rows] * 2)
        asked = K.paged_workspace_bytes(pages.cache, 2 * rows, rows)
        o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows)
        want = [attend(q[b * rows:(b + 1) * rows].double(), stands_for(k[b], fp8), stands_for(v[b], fp8), list(range(first[b], L[b])), p) for b in range(2)]
        o_want, lse_want, o_off, lse_off = (torch.cat(x) for x in zip(*want))
        for size in {0, 16, asked // 2, asked // 5, max(asked - 1, 0), asked, buffer.numel()}:
            buffer.fill_(255)                              # (NaN)
            o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, workspace=buffer[:size])
            assert bool(((o.double() - o_want).abs() <= o_off).all()) and bool(((lse.double() - lse_want).abs() <= lse_off).all()), (rows, size)
            assert bool((buffer[size:] == 255).all())
            if size >= asked:
                assert torch.equal(o.view(torch.int16), o0.view(torch.int16)) and torch.equal(lse, lse0)
            else:
                fewer += 1
                with pytest.raises(K.KsaError):            # the same number of spans, asked for, does not fit
                    K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, workspace=buffer[:size],
                                    n_splits=asked // (2 * rows * 8 * 132 * 4))
    assert fewer >= 8
