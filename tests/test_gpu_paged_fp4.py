"""GPU tests of the 4-bit paged cache: rows in, rows out, and attention over them, against float64 definitions (tests/paged.py, tests/paged_fp4.py)."""
import math

import numpy as np
import pytest
import torch

import paper_2604_24432_amd as K
from tests.paged import attend, batch_of, kinds, mask, randn
from tests.paged_fp4 import Pages4, e2m1, packed
from tests.test_gpu_paged import FEW, LARGE, MANY, bits, say

pytestmark = pytest.mark.gpu


def sequences(p, pages, first, count, seed):
    out = []
    for b in range(p.batch):
        n = first[b] + count[b]
        k, v = randn(n, p.n_kv_heads, p.head_dim, seed=seed + 2 * b), randn(n, p.n_kv_heads, p.head_dim, seed=seed + 2 * b + 1)
        pages.put(b, 0, k, v)
        out.append((e2m1(k.double())[0], e2m1(v.double())[0]))
    return out


def bounds(q, k, v, rows, p):
    """tests.paged.attend, whose bound is relative to every column's own weighted sum, with what that leaves out: a 4-bit column may hold zeros for all keys
    but those of the smallest weights, and 32 bits keep no weight, and no product with a value, below 2^-126.  A row's reference is one of its scores, so its
    weights sum up to 1 at least, and n keys lose n 2^-126 (1 + |v|) at most; 2^7 to spare."""
    want, want_lse, off, lse_off = attend(q, k, v, rows, p)
    return want, want_lse, off + k.shape[0] * 2.0 ** -119 * (1 + float(v.abs().max())), lse_off


def check_attention(p, page, first, count, seed, n_splits=0, max_rows=None, order="phsd", scale_q=1.0, every=1):
    pages = Pages4(p, [a + n for a, n in zip(first, count)], page, seed, order=order)
    seqs = sequences(p, pages, first, count, seed)
    total = sum(count)
    q = (randn(total, p.n_q_heads, p.head_dim, seed=seed + 999).float() * scale_q).to(torch.bfloat16)
    cu, start = batch_of(first, count)
    o, lse = torch.full_like(q, 7.0), torch.full((total, p.n_q_heads), 7.0, device="cuda")
    K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=max_rows, o=o, lse=lse, n_splits=n_splits)
    torch.cuda.synchronize()
    worst, at = 0.0, 0
    for b, n in enumerate(count):
        if n == 0:
            continue
        rows = list(range(0, n, every))
        pick = torch.tensor(rows, device="cuda") + at
        want, want_lse, off, lse_off = bounds(q[pick].double(), *seqs[b], [first[b] + r for r in rows], p)
        err, lse_err = (o[pick].double() - want).abs(), (lse[pick].double() - want_lse).abs()
        assert bool(torch.isfinite(err).all()) and bool(torch.isfinite(lse_err).all()), (b, "not finite")
        worst = max(worst, float((err / off).max()), float((lse_err / lse_off).max()))
        assert bool((err <= off).all()), (b, float((err / off).max()))
        assert bool((lse_err <= lse_off).all()), (b, float((lse_err / lse_off).max()))
        at += n
    say(f"  largest error / bound {worst:.3f}")


def test_every_bf16_value_and_the_ends_of_the_exponents():
    """Each of the 65536 patterns in groups of its own exponents, infinities and NaN among them."""
    say("fp4 every value")
    p = K.make_params(1, 4096, 64, 8, 1, 2, 2, 128)
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(256, 256)      # 2 heads of 128
    g = torch.Generator().manual_seed(3)
    shuffled = x.flatten()[torch.randperm(65536, generator=g)].view(256, 256)
    near = torch.randn(512, 256, generator=g).to(torch.bfloat16)
    halfway = (torch.randint(-28, 29, (512, 256), generator=g) * 0.25 * torch.exp2(torch.randint(-130, 128, (512, 1), generator=g).double())).to(torch.bfloat16)
    zeros = torch.zeros(2, 256, dtype=torch.bfloat16)
    rows = torch.cat([x, x.T.contiguous(), shuffled, near, halfway, zeros]).view(-1, 2, 128).cuda()
    n = rows.shape[0]
    pages = Pages4(p, [n], 64)
    cu, start = batch_of([0], [n])
    K.ksa_paged_append(pages.cache, rows, rows.flip(0).contiguous(), cu, start)
    k, v = K.ksa_paged_read(pages.cache, cu, start, n)
    at, slot = (t.cuda() for t in pages.places(0, 0, n))
    for got, pool, exp, src in ((k, pages.k, pages.k_exp, rows), (v, pages.v, pages.v_exp, rows.flip(0))):
        value, code, e = e2m1(src.double())
        assert torch.equal(exp[at, :, slot], e)
        assert torch.equal(pool[at, :, slot], packed(code))
        assert torch.equal(torch.isnan(got), torch.isnan(value))
        assert torch.equal(got.double().nan_to_num(0.0), value.nan_to_num(0.0))
    assert bool(torch.isnan(k).any()) and bool((k[-1] == 0).all())


MOVES = [(1, 8, 128, 64, 8, 1, 16, [100], [1]), (3, 2, 64, 48, 6, 2, 8, [0, 53, 700], [60, 1, 129]), (4, 5, 128, 8, 1, 3, 32, [9, 0, 77, 8], [0, 17, 300, 5]),
         (2, 1, 64, 1, 0, 15, 128, [40, 3], [33, 90])]


@pytest.mark.parametrize("order", ["phsd", "pshd"])
@pytest.mark.parametrize("case", MOVES, ids=lambda x: "x".join(map(str, x[:7])))
def test_append_and_read(case, order):
    B, Hkv, d, c, m, C, page, first, count = case
    say(f"fp4 moves {case} {order}")
    p = K.make_params(B, 4096, c, m, C, Hkv, Hkv, d)
    pages = Pages4(p, [a + n for a, n in zip(first, count)], page, 5, order=order)
    want = Pages4(p, [a + n for a, n in zip(first, count)], page, 5, order=order)
    total = sum(count)
    wide = randn(total + 2, Hkv + 1, 2, d, seed=4)                     # sources with strides of their own
    k_new, v_new = wide[1:-1, 1:, 0], wide[1:-1, 1:, 1]
    cu, start = batch_of(first, count)
    K.ksa_paged_append(pages.cache, k_new, v_new, cu, start)
    at = 0
    for b, n in enumerate(count):
        want.put(b, first[b], k_new[at:at + n].contiguous(), v_new[at:at + n].contiguous())
        at += n
    for x in ("k", "v", "k_exp", "v_exp"):                             # slots of no row of the call among them
        assert torch.equal(getattr(pages, x), getattr(want, x)), x
    k, v = torch.full((total + 3, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((total + 3, Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    K.ksa_paged_read(pages.cache, cu, start, total + 3, k, v)
    for got, src in ((k, k_new), (v, v_new)):
        assert torch.equal(got[:total].double(), e2m1(src.double())[0])
        assert bool((got[total:] == 7).all())                          # rows behind the last sequence


@pytest.mark.parametrize("case", FEW)
def test_few_rows(case):
    Hq, Hkv, d, c, m, C, page, first, count = case
    say(f"fp4 few rows {case}")
    p = K.make_params(len(first), 4096, c, m, C, Hq, Hkv, d)
    for n_splits in (1, 3, 0):
        check_attention(p, page, first, count, 11, n_splits, max(count))


# every number of pairs of a KV head around the lines between the kernels' columns
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,count", [(1, 1, [1]), (2, 2, [1, 0, 3]), (15, 1, [1, 1]), (16, 1, [1]), (17, 1, [1]), (31, 1, [1]), (32, 1, [1, 1]), (33, 1, [1]), (4, 1, [4, 1]),
                                          (4, 1, [5, 2]), (5, 1, [3, 6]), (8, 8, [16, 1]), (8, 8, [17, 32])])
def test_any_number_of_pairs(Hq, Hkv, count, d):
    say(f"fp4 pairs {Hq}/{Hkv} {count} d={d}")
    first = [333 + 71 * b for b in range(len(count))]
    p = K.make_params(len(count), 2048, 16, 2, 3, Hq, Hkv, d)
    for n_splits in (1, 2):
        check_attention(p, 16, first, count, 31, n_splits, max(count))


@pytest.mark.parametrize("case", MANY)
def test_many_rows(case):
    Hq, Hkv, d, c, m, C, page, first, count = case
    say(f"fp4 many rows {case}")
    p = K.make_params(len(first), 4096, c, m, C, Hq, Hkv, d)
    for n_splits in (1, 3, 0):
        check_attention(p, page, first, count, 12, n_splits)


@pytest.mark.parametrize("case", LARGE)
def test_large_tiles_and_long_lists(case):
    Hq, Hkv, d, c, m, C, page, n_text, first, count = case
    say(f"fp4 large {case}")
    p = K.make_params(len(first), n_text, c, m, C, Hq, Hkv, d)
    check_attention(p, page, first, count, 13)


@pytest.mark.parametrize("rows", [1, 3, 50])
def test_rows_outside_the_heads_and_a_scale_of_its_own(rows):
    say(f"fp4 order and scale {rows}")
    p = K.make_params(1, 1024, 16, 2, 3, 8, 2, 128, softmax_scale=0.3)
    check_attention(p, 16, [200], [rows], 14, order="pshd", scale_q=0.5)


@pytest.mark.parametrize("rows", [1, 40])
def test_summary_rows_that_see_only_themselves(rows):
    say(f"fp4 self only {rows}")
    p = K.make_params(1, 1024, 16, 4, 2, 4, 2, 64, flags=K.KSA_FLAG_SUMMARY_SELF_ONLY)
    check_attention(p, 16, [197], [rows], 15)


@pytest.mark.parametrize("rows", [1, 300])
def test_long_sequences(rows):
    say(f"fp4 long {rows}")
    p = K.make_params(1, 131072, 64, 8, 1, 4, 1, 128)
    n = K.binding.augmented_rows(p, 131072)
    check_attention(p, 64, [n - rows], [rows], 16, every=37 if rows > 1 else 1)


@pytest.mark.parametrize("rows,n_splits", [(1, 1), (8, 1), (8, 2), (150, 1), (150, 3)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_no_number_reaches_a_row_that_does_not_see_it(rows, n_splits, value):
    """A group that is no numbers makes the rows that see it NaN: in K all of a row's output, in V the group's 32 columns."""
    say(f"fp4 no number {rows} splits={n_splits} {value}")
    c, m, C, Hq, Hkv, d, first = 16, 2, 2, 4, 2, 128, 300
    p = K.make_params(1, 2048, c, m, C, Hq, Hkv, d)
    n = first + rows
    see = mask(np.arange(first, n), n, c, m, C)
    for key in (first, first + rows // 2, first - 1, int(np.nonzero(see[0])[0][0])):
        for which in ("k", "v"):
            k, v = randn(n, Hkv, d, seed=1), randn(n, Hkv, d, seed=2)
            q = randn(rows, Hq, d, seed=3)
            cu, start = batch_of([first], [rows])
            out = []
            for bad in (False, True):
                x, y = k.clone(), v.clone()
                if bad:
                    (x if which == "k" else y)[key, 1, 70] = value
                pages = Pages4(p, [n], 16, 7)
                K.ksa_paged_append(pages.cache, x, y, *batch_of([0], [n]))
                out.append(K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=n_splits))
            (o0, lse0), (o, lse) = out
            reached = torch.from_numpy(see[:, key]).cuda()
            hit = torch.zeros_like(o, dtype=torch.bool)
            hit[reached, 2:, :] = True
            if which == "v":
                hit[:, :, :64], hit[:, :, 96:] = False, False
            assert bool(torch.isnan(o[hit]).all()), (key, which)
            assert torch.equal(bits(o)[~hit], bits(o0)[~hit]), (key, which)
            if which == "v":
                assert torch.equal(lse, lse0)
            else:
                assert bool(torch.isnan(lse[reached, 2:]).all()) and torch.equal(lse[~reached], lse0[~reached]) and torch.equal(lse[:, :2], lse0[:, :2])


WILD = [(0, 0x7e), (1, 0xff), (253, 0x77), (254, 0x7f), (255, 0x77), (255, 0x00)]     # exponent bytes outside the format, payloads


@pytest.mark.parametrize("rows,n_splits", [(3, 1), (3, 9), (60, 1), (60, 2)])
def test_slots_never_written_reach_no_row(rows, n_splits):
    """What no row sees may hold any byte: slots behind the last row, summaries that are listed and seen by none."""
    say(f"fp4 wild exponents {rows} splits={n_splits}")
    c, m, C, Hq, Hkv, d = 16, 2, 2, 4, 2, 128
    first = 40 * (c + m) + c - 2
    n = first + rows
    p = K.make_params(1, 4096, c, m, C, Hq, Hkv, d)
    q = randn(rows, Hq, d, seed=3)
    cu, start = batch_of([first], [rows])
    see = mask(np.arange(first, n), n, c, m, C).any(0)
    _, text, idx = kinds(n, c, m)
    unseen = torch.from_numpy(np.nonzero(~see)[0])
    outs = []
    for exponent, byte in WILD:
        pages = Pages4(p, [n], 16, 7, exponent=exponent, byte=byte)
        pages.put(0, 0, randn(n, Hkv, d, seed=1), randn(n, Hkv, d, seed=2))
        at, slot = pages.places(0, 0, n)
        at, slot = at[unseen].cuda(), slot[unseen].cuda()
        for pool, exp in ((pages.k, pages.k_exp), (pages.v, pages.v_exp)):
            pool[at, :, slot], exp[at, :, slot] = byte, exponent
        outs.append(K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=n_splits))
    for o, lse in outs:
        assert bool(torch.isfinite(o.float()).all())
        assert torch.equal(bits(o), bits(outs[0][0])) and torch.equal(lse, outs[0][1])


@pytest.mark.parametrize("rows,n_splits", [(2, 1), (2, 3), (70, 1), (70, 2)])
def test_rows_without_a_page(rows, n_splits):
    say(f"fp4 missing page {rows} splits={n_splits}")
    c, m, C, Hq, Hkv, d, first, page = 16, 2, 2, 4, 2, 64, 500, 8
    p = K.make_params(1, 2048, c, m, C, Hq, Hkv, d)
    n = first + rows
    see = mask(np.arange(first, n), n, c, m, C)
    _, text, idx = kinds(n, c, m)
    cu, start = batch_of([first], [rows])
    q = randn(rows, Hq, d, seed=3)
    for entry in (-1, 10 ** 6):
        for of_text, col in ((True, idx[text][-1] // page), (False, 1)):
            pages = Pages4(p, [n], page, 7, exponent=254)
            pages.put(0, 0, randn(n, Hkv, d, seed=1), randn(n, Hkv, d, seed=2))
            o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=n_splits)
            (pages.text_dev if of_text else pages.sums_dev)[0, col] = entry
            gone = (text == of_text) & (idx // page == col)
            hit = torch.from_numpy(see[:, gone].any(1)).cuda()
            o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=n_splits)
            assert bool(torch.isnan(o[hit]).all()) and bool(torch.isnan(lse[hit]).all()) and bool(hit.any())
            assert torch.equal(bits(o)[~hit], bits(o0)[~hit]) and torch.equal(lse[~hit], lse0[~hit])
            k, _ = K.ksa_paged_read(pages.cache, *batch_of([0], [n]), n)
            assert torch.equal(torch.isnan(k).all(-1).all(-1).cpu(), torch.from_numpy(gone))


def test_pages_further_apart_than_32_bits():
    say("fp4 far pages")
    p = K.make_params(1, 512, 64, 8, 1, 2, 1, 128)
    n = 300
    pages = Pages4(p, [n], 64, 7)
    far = torch.empty(5 << 30, dtype=torch.uint8, device="cuda")                      # pages 1 GiB apart
    used = torch.unique(torch.cat([pages.text.flatten(), pages.sums.flatten()]))
    used = used[used >= 0]
    assert len(used) <= 6
    stride = (5 << 30) // 7 // 64 * 64
    k = torch.as_strided(far, (7, 1, 64, 64), (stride, stride, 64, 1))
    cache = K.PagedCache(p, k, k, *(torch.where(t >= 0, torch.searchsorted(used, t.clamp(min=0)), -1).to(torch.int32).cuda() for t in (pages.text, pages.sums)),
                         torch.zeros(7, 1, 64, 4, dtype=torch.uint8, device="cuda"), torch.zeros(7, 1, 64, 4, dtype=torch.uint8, device="cuda"))
    x = randn(n, 1, 128, seed=1)
    cu, start = batch_of([0], [n])
    K.ksa_paged_append(cache, x, x, cu, start)
    got, _ = K.ksa_paged_read(cache, cu, start, n)
    value = e2m1(x.double())[0]
    assert torch.equal(got.double(), value)
    for rows in (1, 100):
        q = randn(rows, 2, 128, seed=2)
        o, lse = K.ksa_paged_fwd(cache, q, *batch_of([n - rows], [rows]), max_rows=rows)
        want, want_lse, off, lse_off = bounds(q.double(), value, value, list(range(n - rows, n)), p)
        assert bool(((o.double() - want).abs() <= off).all()) and bool(((lse.double() - want_lse).abs() <= lse_off).all())


@pytest.mark.parametrize("rows,n_splits", [(1, 4), (1, 1), (40, 3)])
def test_graph_replays_and_repeated_calls(rows, n_splits):
    """Append and attention in a graph, replayed with other rows, places and pages, eager work in between: the eager calls' bits."""
    say(f"fp4 graph {rows} splits={n_splits}")
    p = K.make_params(2, 2048, 16, 2, 3, 8, 2, 128)
    pages = Pages4(p, [900, 900], 16, 3)
    for b in range(2):
        pages.put(b, 0, randn(900, 2, 128, seed=b), randn(900, 2, 128, seed=b + 5))
    k, v, q = randn(2 * rows, 2, 128, seed=21), randn(2 * rows, 2, 128, seed=22), randn(2 * rows, 8, 128, seed=23)
    cu, start = batch_of([500, 700], [rows, rows])
    ws = torch.empty(K.paged_workspace_bytes(pages.cache, 2 * rows, rows, n_splits), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(2 * rows, 8, device="cuda")

    def step():
        K.ksa_paged_append(pages.cache, k, v, cu, start)
        K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, o=o, lse=lse, workspace=ws, n_splits=n_splits)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for r in range(4):
        k.copy_(randn(2 * rows, 2, 128, seed=31 + r)), q.copy_(randn(2 * rows, 8, 128, seed=41 + r))
        start.copy_(torch.tensor([500 + 13 * r, 700 - 29 * r], dtype=torch.int32))
        pages.text_dev.copy_(pages.text_dev[:, torch.randperm(pages.text.shape[1], generator=torch.Generator().manual_seed(r)).cuda()])
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        o.zero_(), lse.zero_()
        for _ in range(2):
            step()
            assert torch.equal(bits(o), bits(got[0])) and torch.equal(lse, got[1])


def test_a_prompt_in_pieces_then_tokens_agree_with_the_bf16_cache():
    """The attention over a 4-bit cache is that of a bf16 cache holding the rows that ksa_paged_read gives."""
    say("fp4 against bf16 cache")
    p = K.make_params(1, 2048, 64, 8, 1, 32, 8, 128)
    n = 700
    pages = Pages4(p, [n], 16, 3)
    k, v, q = randn(n, 8, 128, seed=1), randn(n, 8, 128, seed=2), randn(n, 32, 128, seed=3)
    at = 0
    for piece in (333, 200, 1, 1, 1, 164):
        K.ksa_paged_append(pages.cache, k[at:at + piece], v[at:at + piece], *batch_of([at], [piece]))
        at += piece
    kb, vb = K.ksa_paged_read(pages.cache, *batch_of([0], [n]), n)
    plain = torch.zeros(pages.k.shape[0], 8, 16, 128, dtype=torch.bfloat16, device="cuda")
    other = K.PagedCache(p, plain, plain.clone(), pages.text_dev, pages.sums_dev)
    K.ksa_paged_append(other, kb, vb, *batch_of([0], [n]))
    for first, rows in ((n - 1, 1), (n - 7, 7), (100, 600)):
        x, y = (K.ksa_paged_fwd(c, q[first:first + rows], *batch_of([first], [rows]), max_rows=rows) for c in (pages.cache, other))
        want = bounds(q[first:first + rows].double(), kb.double(), vb.double(), list(range(first, first + rows)), p)
        for got in (x, y):
            assert bool(((got[0].double() - want[0]).abs() <= want[2]).all()) and bool(((got[1].double() - want[1]).abs() <= want[3]).all())


def test_python_refuses_what_does_not_fit():
    p = K.make_params(1, 512, 64, 8, 1, 2, 1, 128)
    pages = Pages4(p, [100], 16, 3)
    k, e = pages.k, pages.k_exp
    text, sums = pages.text_dev, pages.sums_dev
    for bad in ((k, k, text, sums), (k, k, text, sums, e), (k, k, text, sums, None, e), (k[..., :32], k[..., :32], text, sums, e, e), (k, k, text, sums, e[..., :2], e[..., :2]),
                (k, k, text, sums, e[..., 0], e[..., 0]), (k, k.to(torch.bfloat16), text, sums, e, e), (k, k, text, sums, e.int(), e.int())):
        with pytest.raises(ValueError):
            K.PagedCache(p, *bad)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 5])
def test_more_workgroups_than_places(d, rows):
    """Beyond 512 workgroups of few rows, where those of four waves take over; 16 and 32 columns of pairs, sequences of many lengths, some without rows."""
    say(f"fp4 many workgroups d={d} rows={rows}")
    B = 140
    p = K.make_params(B, 1024, 16, 2, 3, 16, 4, d)
    first, count = [(37 * b) % 190 for b in range(B)], [rows if b % 7 else b % 2 for b in range(B)]
    for n_splits in (1, 2):
        check_attention(p, 16, first, count, 41, n_splits, rows)


@pytest.mark.parametrize("rows", [1, 4, 70])
@pytest.mark.parametrize("n_splits", [1, 2])
def test_sequences_out_of_place(rows, n_splits):
    """A sequence that starts outside the text, has more rows than were said, or borders outside the tensor: NaN for its rows, the others as they were."""
    say(f"fp4 out of place rows={rows} splits={n_splits}")
    p = K.make_params(4, 300, 16, 2, 2, 8, 2, 128)
    pages = Pages4(p, [200] * 4, 16, 3)
    for b in range(4):
        pages.put(b, 0, randn(200, 2, 128, seed=b), randn(200, 2, 128, seed=b + 9))
    total = 4 * rows
    q = randn(total + 3, 8, 128, seed=5)
    cu = torch.arange(5, dtype=torch.int32, device="cuda") * rows
    start = torch.full((4,), 100, dtype=torch.int32, device="cuda")

    def run(cu, start, max_rows=rows):
        o, lse = torch.full_like(q, 7.0), torch.full((total + 3, 8), 7.0, device="cuda")
        K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=max_rows, o=o, lse=lse, n_splits=n_splits)
        return o, lse

    good = run(cu, start)
    assert bool(torch.isfinite(good[0][:total].float()).all()) and bool((good[0][total:] == 7).all()) and bool((good[1][total:] == 7).all())
    for bad in (-1, 10 ** 6, 338 - rows + 1):                              # 300 text tokens have 336 rows
        at = start.clone()
        at[2] = bad
        for got, want in zip(run(cu, at), good):
            assert bool(torch.isnan(got[2 * rows:3 * rows]).all())
            assert torch.equal(got[:2 * rows], want[:2 * rows]) and torch.equal(got[3 * rows:], want[3 * rows:])


def test_a_stream_of_its_own():
    say("fp4 stream")
    p = K.make_params(2, 2048, 16, 2, 3, 8, 2, 128)
    pages = Pages4(p, [900, 900], 16, 3)
    k, v, q = randn(1800, 2, 128, seed=1), randn(1800, 2, 128, seed=2), randn(2, 8, 128, seed=3)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    K.ksa_paged_append(pages.cache, k, v, *batch_of([0, 0], [900, 900]), stream=stream)
    o, lse = K.ksa_paged_fwd(pages.cache, q, *batch_of([899, 899], [1, 1]), max_rows=1, stream=stream)
    kb, _ = K.ksa_paged_read(pages.cache, *batch_of([0, 0], [900, 900]), 1800, stream=stream)
    stream.synchronize()
    assert torch.equal(kb.double(), e2m1(k.double())[0])
    o1, lse1 = K.ksa_paged_fwd(pages.cache, q, *batch_of([899, 899], [1, 1]), max_rows=1)
    assert torch.equal(bits(o), bits(o1)) and torch.equal(lse, lse1)


@pytest.mark.parametrize("rows,n_splits", [(1, 1), (1, 3), (6, 1), (60, 1), (60, 2)])
def test_outputs_in_the_queries_place_and_strided(rows, n_splits):
    say(f"fp4 in place rows={rows} splits={n_splits}")
    p = K.make_params(3, 2048, 16, 2, 3, 8, 2, 128)
    pages = Pages4(p, [900] * 3, 16, 3)
    for b in range(3):
        pages.put(b, 0, randn(900, 2, 128, seed=b), randn(900, 2, 128, seed=b + 9))
    q = randn(3 * rows, 8, 128, seed=5)
    cu, start = batch_of([500, 899 - rows, 0], [rows] * 3)
    o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=n_splits)
    x = q.clone()
    K.ksa_paged_fwd(pages.cache, x, cu, start, max_rows=rows, n_splits=n_splits, o=x, return_lse=False)
    assert torch.equal(bits(x), bits(o))
    wide = torch.full((3 * rows, 3, 10, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 0, :8] = q
    K.ksa_paged_fwd(pages.cache, wide[:, 0, :8], cu, start, max_rows=rows, n_splits=n_splits, o=wide[:, 2, 1:9], return_lse=False)
    assert torch.equal(bits(wide[:, 2, 1:9]), bits(o)) and torch.equal(bits(wide[:, 0, :8]), bits(q))
    assert bool((wide[:, 1] == 7).all()) and bool((wide[:, 2, 0] == 7).all()) and bool((wide[:, 2, 9] == 7).all())


@pytest.mark.parametrize("rows", [1, 60])
def test_products_that_overflow_before_they_are_scaled(rows):
    """q k beyond 3.4e38 whose scaled scores are not: the power of two of the scale that goes into q keeps them finite."""
    say(f"fp4 large products {rows}")
    d = 128
    p = K.make_params(1, 1024, 16, 2, 3, 4, 2, d, softmax_scale=2.0 ** -8)
    pages = Pages4(p, [300], 16, 3)
    k, v = randn(300, 2, d, seed=1), randn(300, 2, d, seed=2)
    big = torch.zeros_like(k)
    big[..., 0] = k[..., 0].sign() * 2.0 ** 63                          # one element each: q k = +- 2^132 before, +- 2^124 after the scale
    big[150:, :, 0] = 0.0
    pages.put(0, 0, big, v)
    q = torch.zeros(rows, 4, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 2.0 ** 69
    first = 300 - rows
    o, lse = K.ksa_paged_fwd(pages.cache, q, *batch_of([first], [rows]), max_rows=rows)
    kk, vv = e2m1(big.double())[0], e2m1(v.double())[0]
    see = torch.from_numpy(mask(np.arange(first, 300), 300, 16, 2, 3)).cuda()
    for h in range(4):
        s = (q[:, h].double() @ kk[:, h // 2].T * 2.0 ** -8).masked_fill(~see, -math.inf)
        want = torch.softmax(s, 1) @ vv[:, h // 2]
        assert bool(torch.isfinite(o[:, h].float()).all()) and bool(torch.isfinite(lse[:, h]).all())
        # equal scores have equal weights: the mean of some values, to the roundings of bf16 (weights of 1, the output) and of 300 sums
        assert bool(((o[:, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + 300 * 2.0 ** -24 * float(vv.abs().max())).all()), h


# pages, of which the last ones are used, every gap-th; bytes from page to page
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_pages,gap,stride", [(8, 1, 1 << 30), ((1 << 25) + 200, 16, 272)], ids=["1 GiB apart", "exponents beyond 4 GiB"])
def test_rows_and_exponents_beyond_32_bits(n_pages, gap, stride, d):
    """Pools and exponents larger than 4 GiB: every byte where it belongs, by append and by the rotary call, and found there by all that reads.  (The pages lie
    closer to each other than they are long, where only every 16th is used.)"""
    say(f"fp4 beyond 32 bits {n_pages} {stride} d={d}")
    page, n, c, m = 64, 300, 64, 8
    p = K.make_params(1, 512, c, m, 1, 2, 1, d)
    cols = K.paged_pages(p, page, n)
    used = [n_pages - 1 - gap * x for x in range(sum(cols))]
    assert min(used) >= 0 and max(used) * stride >= 2 ** 32 and (gap == 1 or min(used) * page * (d // 32) >= 2 ** 32) and gap * stride >= page * d // 2
    text, sums = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (used[:cols[0]], used[cols[0]:]))

    def pool():
        far = torch.empty((n_pages - 1) * stride + page * d // 2, dtype=torch.uint8, device="cuda")
        return torch.as_strided(far, (n_pages, 1, page, d // 2), (stride, page * d // 2, d // 2, 1))

    pools, exps = [pool(), pool()], [torch.zeros(n_pages, 1, page, d // 32, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = K.PagedCache(p, *pools, text, sums, *exps)
    _, is_text, idx = kinds(n, c, m)
    at = torch.tensor([(used[:cols[0]] if t else used[cols[0]:])[i // page] for t, i in zip(is_text, idx)], device="cuda")
    slot = torch.from_numpy(idx % page).cuda()
    cu, start = batch_of([0], [n])
    k, v = randn(n, 1, d, seed=1), randn(n, 1, d, seed=2)

    def holds(*rows):
        for x, pool_of, exp_of in zip(rows, pools, exps):
            _, code, e = e2m1(x.double())
            assert torch.equal(pool_of[at, :, slot], packed(code)) and torch.equal(exp_of[at, :, slot], e)

    rotary, line = K.Rotary(d), torch.zeros(1, K.binding.augmented_rows(p, 512), 1, d, dtype=torch.bfloat16, device="cuda")
    line[0, :n] = k
    K.ksa_paged_rotary(cache, rotary, None, k, v, cu, start)
    holds(K.ksa_rotary_fwd(p, rotary, None, line)[1][0, :n], v)
    K.ksa_paged_append(cache, k, v, cu, start)
    holds(k, v)
    value = [e2m1(x.double())[0] for x in (k, v)]
    for got, want in zip(K.ksa_paged_read(cache, cu, start, n), value):
        assert torch.equal(got.double(), want)
    for rows in (1, 10, 100):                                             # 2 and 20 pairs of rows and heads, then tiles of them
        q = randn(rows, 2, d, seed=3)
        o, lse = K.ksa_paged_fwd(cache, q, *batch_of([n - rows], [rows]), max_rows=rows)
        want, want_lse, off, lse_off = bounds(q.double(), *value, list(range(n - rows, n)), p)
        assert bool(((o.double() - want).abs() <= off).all()) and bool(((lse.double() - want_lse).abs() <= lse_off).all()), rows
