"""GPU tests of the paged cache: rows in, rows out, and attention over them, against float64 definitions (tests/paged.py)."""
import math
import sys

import numpy as np
import pytest
import torch

import paper_2604_24432_amd as K
from tests.paged import Pages, attend, batch_of, e4m3, randn, stands_for

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def bits(t):
    return t.contiguous().view(torch.int16)


def check_attention(p, page, fp8, first, count, seed, n_splits=0, max_rows=None, order="phsd", scale_q=1.0):
    B, Hkv, d = p.batch, p.n_kv_heads, p.head_dim
    pages = Pages(p, [a + n for a, n in zip(first, count)], page, fp8, seed, order=order)
    seqs = []
    for b in range(B):
        k, v = randn(first[b] + count[b], Hkv, d, seed=seed + 2 * b), randn(first[b] + count[b], Hkv, d, seed=seed + 2 * b + 1)
        pages.put(b, 0, k, v)
        seqs.append((k, v))
    total = sum(count)
    q = (randn(total, p.n_q_heads, d, seed=seed + 999).float() * scale_q).to(torch.bfloat16)
    cu, start = batch_of(first, count)
    o, lse = torch.full_like(q, 7.0), torch.full((total, p.n_q_heads), 7.0, device="cuda")
    K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=max_rows, o=o, lse=lse, n_splits=n_splits)
    torch.cuda.synchronize()
    worst, at = 0.0, 0
    for b in range(B):
        n = count[b]
        if n == 0:
            continue
        k, v = (stands_for(x, fp8) for x in seqs[b])
        want, want_lse, off, lse_off = attend(q[at:at + n].double(), k, v, list(range(first[b], first[b] + n)), p)
        err, lse_err = (o[at:at + n].double() - want).abs(), (lse[at:at + n].double() - want_lse).abs()
        assert bool(torch.isfinite(err).all()) and bool(torch.isfinite(lse_err).all()), (b, "not finite")
        worst = max(worst, float((err / off).max()), float((lse_err / lse_off).max()))
        assert bool((err <= off).all()), (b, float((err / off).max()))
        assert bool((lse_err <= lse_off).all()), (b, float((lse_err / lse_off).max()))
        at += n
    say(f"  largest error / bound {worst:.3f}")


# (heads, kv_heads, d, c, m, C, page, first new row, new rows)
FEW = [
    (8, 1, 64, 8, 1, 32, 16, [786], [1]),
    (32, 8, 128, 64, 8, 1, 64, [0, 1, 63, 64, 71, 72], [1] * 6),                 # the first rows, a summary row, a new chunk
    (4, 4, 128, 64, 8, 1, 16, [700, 71, 215, 2000], [1] * 4),
    (12, 4, 64, 48, 6, 2, 8, [1500, 53, 160], [5, 2, 4]),                        # text and summary rows together, short pages
    (16, 1, 128, 8, 1, 4, 32, [333, 80], [2, 1]),
    (16, 2, 64, 16, 2, 3, 16, [100, 17, 0], [4, 3, 2]),
    (32, 1, 64, 20, 5, 2, 64, [477], [1]),
    (7, 1, 128, 1, 0, 15, 8, [40, 3], [4, 4]),                                   # a sliding window, seven heads
    (2, 1, 128, 64, 0, 4096, 128, [1111, 127], [16, 1]),                         # full attention
    (6, 2, 64, 8, 8, 0, 16, [203, 8], [8, 9]),                                   # as many summaries as text, no window
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", FEW)
def test_few_rows(case, fp8):
    Hq, Hkv, d, c, m, C, page, first, count = case
    say(f"paged few rows {case} fp8={fp8}")
    p = K.make_params(len(first), 4096, c, m, C, Hq, Hkv, d)
    for n_splits in (1, 3, 0):
        check_attention(p, page, fp8, first, count, 11, n_splits, max(count))


MANY = [
    (8, 2, 64, 64, 8, 1, 16, [100], [200]),
    (32, 8, 128, 64, 8, 1, 64, [0, 500, 71], [150, 9, 33]),
    (4, 4, 128, 64, 8, 1, 32, [1000], [129]),
    (12, 4, 64, 48, 6, 2, 8, [1500, 53, 160, 7], [77, 0, 301, 1]),
    (40, 1, 128, 8, 1, 4, 32, [333, 80], [20, 1]),
    (16, 2, 64, 16, 2, 3, 16, [100, 17], [65, 6]),
    (3, 1, 128, 1, 0, 15, 8, [40, 3], [90, 44]),
    (2, 1, 128, 64, 0, 4096, 128, [1111, 127], [300, 64]),
    (6, 2, 64, 8, 8, 0, 16, [203, 8], [160, 90]),
    (1, 1, 64, 128, 16, 1, 1024, [0], [1000]),
    (200, 1, 64, 8, 1, 2, 8, [30], [3]),                                         # more heads than a tile has pairs
    (32, 2, 128, 64, 8, 1, 16, [333, 0, 71], [1100, 900, 201]),                  # 65536 pairs and more: larger tiles
    (64, 64, 64, 48, 6, 2, 64, [10, 700], [900, 311]),
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", MANY)
def test_many_rows(case, fp8):
    Hq, Hkv, d, c, m, C, page, first, count = case
    say(f"paged many rows {case} fp8={fp8}")
    p = K.make_params(len(first), 4096, c, m, C, Hq, Hkv, d)
    for n_splits in (1, 3, 0):
        check_attention(p, page, fp8, first, count, 12, n_splits)


# (..., text tokens to reckon with, first new row, new rows): enough rows and keys for the largest query tiles, and few rows with many keys
LARGE = [
    (32, 2, 128, 64, 0, 4096, 32, 4096, [333, 0], [1100, 1000]),
    (32, 4, 64, 64, 0, 4096, 16, 4096, [100], [2100]),
    (30, 3, 128, 16, 4, 8, 16, 16384, [700, 0, 50, 400], [1000, 1, 900, 801]),
    (48, 4, 64, 16, 4, 8, 64, 16384, [700, 0, 3], [1000, 900, 201]),
    (32, 2, 128, 1, 0, 700, 16, 4096, [1000, 30], [1200, 1000]),
    (4, 4, 128, 1, 0, 900, 8, 4096, [1500, 30], [300, 177]),
    (4, 2, 64, 16, 4, 8, 16, 16384, [3500, 0], [100, 90]),
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", LARGE)
def test_large_tiles_and_long_lists(case, fp8):
    Hq, Hkv, d, c, m, C, page, n, first, count = case
    say(f"paged large tiles {case} fp8={fp8}")
    p = K.make_params(len(first), n, c, m, C, Hq, Hkv, d)
    for n_splits in (1, 2, 0):
        check_attention(p, page, fp8, first, count, 18, n_splits, max(count))


@pytest.mark.parametrize("rows", [1, 40])
def test_summary_rows_that_see_only_themselves(rows):
    say(f"paged self-only rows={rows}")
    p = K.make_params(2, 2048, 16, 4, 2, 8, 2, 64, flags=K.KSA_FLAG_SUMMARY_SELF_ONLY)
    check_attention(p, 16, False, [57, 18], [rows, rows], 13)


@pytest.mark.parametrize("rows", [1, 3, 50])
@pytest.mark.parametrize("fp8", [False, True])
def test_rows_outside_the_heads_and_a_scale_of_its_own(rows, fp8):
    say(f"paged strides rows={rows} fp8={fp8}")
    p = K.make_params(2, 2048, 64, 8, 1, 8, 2, 128, softmax_scale=0.3)
    check_attention(p, 32, fp8, [300, 900], [rows, rows], 14, order="pshd")


@pytest.mark.parametrize("rows", [1, 60])
def test_products_that_overflow_before_they_are_scaled(rows):
    """q.k reaches 1e39 while the scaled scores are representable: with all keys alike the weights are uniform."""
    say(f"paged large products rows={rows}")
    p = K.make_params(1, 512, 64, 0, 64, 4, 1, 128)
    n = 200 + rows
    pages = Pages(p, [n], 16, False, 3)
    k = torch.full((n, 1, 128), 2.0 ** 62, device="cuda").to(torch.bfloat16)
    v = randn(n, 1, 128, seed=5)
    pages.put(0, 0, k, v)
    q = torch.full((rows, 4, 128), 2.0 ** 60, device="cuda").to(torch.bfloat16)
    cu, start = batch_of([200], [rows])
    o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start)
    want, want_lse, off, _ = attend(q.double(), k.double(), v.double(), list(range(200, n)), p)
    # (every product is the same power of two and every sum of them exact: equal scores, the weights 1)
    assert bool(((o.double() - want).abs() <= off).all())
    assert bool(((lse.double() - want_lse).abs() <= 2.0 ** -20 * want_lse.abs()).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows", [1, 300])
def test_long_sequences(rows, fp8):
    """Positions around 100 000 in the benchmark's chunk shape; float64 on the GPU."""
    say(f"paged long rows={rows} fp8={fp8}")
    p = K.make_params(1, 131072, 64, 8, 1, 8, 2, 128)
    check_attention(p, 64, fp8, [112345], [rows], 15)


# ---- rows in and out ----------------------------------------------------------------------------------------------------

MOVES = [
    (1, 64, 8, 1, 16, [0], [1]),
    (8, 128, 64, 8, 64, [0, 100, 71], [300, 1, 75]),
    (3, 64, 48, 6, 8, [53, 0, 7, 160], [3, 0, 200, 1]),
    (16, 128, 1, 0, 32, [5, 0], [70, 33]),
    (5, 128, 8, 8, 1024, [0], [777]),
]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("case", MOVES)
def test_append_and_read(case, fp8):
    Hkv, d, c, m, page, first, count = case
    say(f"paged append / read {case} fp8={fp8}")
    p = K.make_params(len(first), 4096, c, m, 1, Hkv, Hkv, d)
    ends = [a + n for a, n in zip(first, count)]
    pages, other = Pages(p, ends, page, fp8, 1, fill=3.0), Pages(p, ends, page, fp8, 1, fill=3.0)
    total = sum(count)
    k, v = randn(total + 5, Hkv, d, seed=2), randn(total + 5, Hkv, d, seed=3)
    if fp8:
        k[0, 0] = 0.0
        k[total // 2, 0, 3], v[total // 2, 0, 1], v[total // 2, 0, 60] = math.inf, math.nan, -math.inf
        v[total - 1, Hkv - 1] = math.nan
    cu, start = batch_of(first, count)
    K.ksa_paged_append(pages.cache, k, v, cu, start)       # (five rows behind the last sequence's)
    at = 0
    for b, n in enumerate(count):
        if n:
            other.put(b, first[b], k[at:at + n], v[at:at + n])
        at += n
    torch.cuda.synchronize()
    for x in ("k", "v"):
        mine, want = getattr(pages, x), getattr(other, x)
        if fp8:
            assert torch.equal(getattr(pages, x + "_exp"), getattr(other, x + "_exp"))
            assert torch.equal(mine.float().nan_to_num(nan=9999.0), want.float().nan_to_num(nan=9999.0))
        else:
            assert torch.equal(bits(mine), bits(want))
    k2, v2 = torch.full_like(k, 5.0), torch.full_like(v, 5.0)
    K.ksa_paged_read(pages.cache, cu, start, total + 5, k=k2, v=v2)
    for mine, x in ((k2, k), (v2, v)):
        want = stands_for(x[:total], fp8)
        assert torch.equal(mine[:total].double().nan_to_num(nan=9999.0), want.nan_to_num(nan=9999.0))
        assert bool((mine[total:] == 5.0).all())


def test_every_finite_bf16_value_and_the_ends_of_the_exponents():
    """All finite bf16 numbers as rows of 64 equal or neighbouring magnitudes, and rows whose largest element lies on either side of 448 * 2^e."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = x[torch.isfinite(x.float())]
    x = torch.cat([x, x[:(-x.numel()) % 64]]).view(-1, 1, 64)
    mixed = x.clone()
    mixed[:, :, ::2] = x.flip(0)[:, :, ::2]                # small beside large
    edge = torch.zeros(40, 1, 64, dtype=torch.bfloat16)
    for i in range(20):
        edge[i, 0, 0], edge[i, 0, 1:] = 1.75 * 2.0 ** (i - 10), 2.0 ** (i - 20)
        edge[20 + i, 0, 0], edge[20 + i, 0, 1:] = (1.75 + 2.0 ** -7) * 2.0 ** (i - 10), 2.0 ** (i - 20)
    rows = torch.cat([x, mixed, edge]).cuda()
    p = K.make_params(1, 65536, 64, 8, 1, 1, 1, 64)
    pages = Pages(p, [rows.shape[0]], 64, True, 1)
    cu, start = batch_of([0], [rows.shape[0]])
    K.ksa_paged_append(pages.cache, rows, rows, cu, start)
    k, v = K.ksa_paged_read(pages.cache, cu, start, rows.shape[0])
    want, _ = e4m3(rows.double())
    assert torch.equal(k.double(), want) and torch.equal(v.double(), want)
    kept = want != 0
    assert bool((k.float()[kept].abs() >= 2.0 ** -126).all())     # normal bf16 numbers


def test_strided_sources_and_outputs():
    p = K.make_params(2, 1024, 64, 8, 1, 4, 2, 128)
    pages = Pages(p, [200, 200], 16, False, 1)
    big = randn(100, 6, 128, seed=1)
    k, v = big[:, 0:4:2], big[:, 1:5:2]                    # head stride 2 d
    cu, start = batch_of([20, 71], [60, 40])
    K.ksa_paged_append(pages.cache, k, v, cu, start)
    out = torch.full((100, 4, 128), 5.0, device="cuda").to(torch.bfloat16)
    K.ksa_paged_read(pages.cache, cu, start, 100, k=out[:, 0::2], v=out[:, 1::2])
    assert torch.equal(bits(out[:, 0::2]), bits(k)) and torch.equal(bits(out[:, 1::2]), bits(v))
    # attention with q in a fused tensor and o in place of it
    first = randn(20, 2, 128, seed=8)
    pages.put(0, 0, first, first)
    pages.put(1, 0, randn(71, 2, 128, seed=9), randn(71, 2, 128, seed=10))
    qkv = randn(100, 8, 128, seed=4)
    q = qkv[:, 2:6]
    o1, lse1 = K.ksa_paged_fwd(pages.cache, q.contiguous(), cu, start)
    rest = qkv.clone()
    o2, lse2 = K.ksa_paged_fwd(pages.cache, q, cu, start, o=q)
    assert torch.equal(bits(o1), bits(o2)) and torch.equal(lse1, lse2)
    assert torch.equal(bits(qkv[:, :2]), bits(rest[:, :2])) and torch.equal(bits(qkv[:, 6:]), bits(rest[:, 6:]))


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_any_number_of_spans(rows):
    """More spans than keys have blocks, up to the most there may be: the same outputs."""
    say(f"paged spans rows={rows}")
    p = K.make_params(2, 4096, 64, 8, 1, 6, 2, 64)
    for n_splits in (2, 4, 5, 8, 9, 63, 64, 65, 130, 1024):
        check_attention(p, 16, n_splits % 2 == 0, [2777, 100], [rows, rows], 16, n_splits, rows)
    p = K.make_params(1, 4096, 64, 8, 1, 3, 1, 128)
    for n_splits in (4, 8, 9, 100):
        check_attention(p, 16, False, [2777], [rows], 17, n_splits, rows)


def test_calls_without_rows():
    """No rows at all, and none that belong to a sequence: nothing is touched."""
    p = K.make_params(2, 1024, 16, 2, 1, 2, 1, 64)
    pages = Pages(p, [100, 50], 8, False, 5, fill=3.0)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cu, start = batch_of([10, 20], [0, 0])
    K.ksa_paged_append(pages.cache, none[:, :1], none[:, :1], cu, start)
    k, v = K.ksa_paged_read(pages.cache, cu, start, 0)
    o, lse = K.ksa_paged_fwd(pages.cache, none, cu, start)
    assert k.shape == v.shape == (0, 1, 64) and o.shape == (0, 2, 64) and lse.shape == (0, 2)
    before = pages.k.clone()
    for rows in (1, 90):
        k, v = torch.full((rows, 1, 64), 5.0, device="cuda").to(torch.bfloat16), torch.full((rows, 1, 64), 6.0, device="cuda").to(torch.bfloat16)
        K.ksa_paged_append(pages.cache, k, v, cu, start)
        K.ksa_paged_read(pages.cache, cu, start, rows, k=k, v=v)
        assert bool((k == 5).all()) and bool((v == 6).all()) and torch.equal(pages.k, before)
        for n_splits in (1, 3, 12):
            o, lse = torch.full((rows, 2, 64), 5.0, device="cuda").to(torch.bfloat16), torch.full((rows, 2), 6.0, device="cuda")
            K.ksa_paged_fwd(pages.cache, o, cu, start, o=o, lse=lse, n_splits=n_splits)
            assert bool((o == 5).all()) and bool((lse == 6).all())


# ---- what may not reach a row -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows,n_splits", [(1, 1), (8, 1), (8, 2), (150, 1), (150, 3)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_no_number_reaches_a_row_that_does_not_see_it(rows, n_splits, value, fp8):
    """A K or V row that is no number: rows that see it are none either, all others keep their bits."""
    say(f"paged no numbers rows={rows} splits={n_splits} {value} fp8={fp8}")
    p = K.make_params(1, 1024, 16, 2, 2, 4, 2, 64)
    first = 233
    n = first + rows
    pages = Pages(p, [n], 8, fp8, 5)
    k, v = randn(n, 2, 64, seed=6), randn(n, 2, 64, seed=7)
    q = randn(rows, 4, 64, seed=8)
    cu, start = batch_of([first], [rows])
    from tests.paged import mask
    see = mask(np.arange(first, n), n, 16, 2, 2)

    def run():
        return K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=n_splits)

    pages.put(0, 0, k, v)
    o0, lse0 = run()
    assert bool(torch.isfinite(o0.float()).all())
    for at in (n - 1, n - 1 - rows // 2, first - 3, 17):
        sees = torch.from_numpy(see[:, at]).cuda()
        k2, v2 = k.clone(), v.clone()
        k2[at, 0, 5] = value
        pages.put(0, 0, k2, v)
        o, lse = run()
        assert torch.equal(bits(o[~sees]), bits(o0[~sees])) and torch.equal(lse[~sees], lse0[~sees])
        assert torch.equal(bits(o[:, 2:]), bits(o0[:, 2:]))                       # the other KV head's
        if not math.isinf(value) or fp8:                                          # (an infinity may give a weight of zero)
            assert bool(torch.isnan(o[sees][:, :2].float()).all()) and bool(torch.isnan(lse[sees][:, :2]).all())
        v2[at, 1, 33] = value
        pages.put(0, 0, k, v2)
        o, lse = run()
        assert torch.equal(bits(o[~sees]), bits(o0[~sees])) and torch.equal(lse, lse0)
        assert not bool(torch.isfinite(o[sees][:, 2:, 33].float()).any())
        o[:, 2:, 33] = o0[:, 2:, 33]
        assert torch.equal(bits(o), bits(o0))                                     # the other columns


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,rows", [(64, 2, 128, 1100), (4, 2, 128, 300), (64, 2, 64, 1100), (4, 2, 64, 300)])
def test_no_number_and_no_page_in_large_tiles(heads, kv_heads, d, rows, fp8):
    """As above and below, in the largest query tiles and where two groups of waves share the keys."""
    say(f"paged no numbers, large tiles {heads}/{kv_heads} d={d} rows={rows} fp8={fp8}")
    p = K.make_params(1, 16384, 16, 2, 2, heads, kv_heads, d)
    first = 1233
    n = first + rows
    pages = Pages(p, [n], 8, fp8, 5)
    k, v = randn(n, kv_heads, d, seed=6), randn(n, kv_heads, d, seed=7)
    q = randn(rows, heads, d, seed=8)
    cu, start = batch_of([first], [rows])
    from tests.paged import kinds, mask
    see = mask(np.arange(first, n), n, 16, 2, 2)
    G = heads // kv_heads
    pages.put(0, 0, k, v)
    o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=1)
    assert bool(torch.isfinite(o0.float()).all())
    for at, of_v in ((n - 1 - rows // 2, False), (n - rows // 3, True), (first - 3, True), (17, True)):
        sees = torch.from_numpy(see[:, at]).cuda()
        bad = (v if of_v else k).clone()
        bad[at, 0, 5] = math.nan
        pages.put(0, 0, *((k, bad) if of_v else (bad, v)))
        o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=1)
        assert torch.equal(bits(o[:, G:]), bits(o0[:, G:])) and torch.equal(lse[:, G:], lse0[:, G:])
        assert torch.equal(bits(o[~sees]), bits(o0[~sees])) and torch.equal(lse[~sees], lse0[~sees])
        if of_v:
            assert bool(torch.isnan(o[sees][:, :G, 5].float()).all()) and torch.equal(lse, lse0)
            rest = [x for x in range(d) if x != 5]
            assert torch.equal(bits(o[:, :, rest]), bits(o0[:, :, rest]))
        else:
            assert bool(torch.isnan(o[sees][:, :G].float()).all()) and bool(torch.isnan(lse[sees][:, :G]).all())
    pages.put(0, 0, k, v)
    _, text, idx = kinds(n, 16, 2)
    for of_text in (True, False):
        page = int(idx[n - rows // 2]) // 8 if of_text else 3
        gone = text & (idx // 8 == page) if of_text else ~text & (idx // 8 == page)
        table, host = (pages.text_dev, pages.text) if of_text else (pages.sums_dev, pages.sums)
        table[0, page] = -1
        o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=1)
        table.copy_(host)
        sees = torch.from_numpy((see & gone).any(1)).cuda()
        assert bool(torch.isnan(o[sees].float()).all()) and bool(torch.isnan(lse[sees]).all())
        assert torch.equal(bits(o[~sees]), bits(o0[~sees])) and torch.equal(lse[~sees], lse0[~sees])


@pytest.mark.parametrize("fp8", [False, True])
def test_rows_without_a_page(fp8):
    say(f"paged missing pages fp8={fp8}")
    p = K.make_params(1, 1024, 16, 2, 1, 2, 1, 64)
    n = 18 * 20
    pages = Pages(p, [n], 8, fp8, 5, fill=1.0)
    k, v = randn(n, 1, 64, seed=6), randn(n, 1, 64, seed=7)
    from tests.paged import kinds, mask
    j, text, idx = kinds(n, 16, 2)
    for bad in (-1, pages.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        # text page 33 (rows 264 .. 271, chunk 16) and summary page 2 (ordinals 16 .. 23)
        tables = pages.text.clone(), pages.sums.clone()
        tables[0][0, 33], tables[1][0, 2] = bad, bad
        pages.text_dev.copy_(tables[0]), pages.sums_dev.copy_(tables[1])
        gone = np.where(text, (idx // 8) == 33, (idx // 8) == 2)
        cu, start = batch_of([0], [n])
        K.ksa_paged_append(pages.cache, k, v, cu, start)
        k2, v2 = K.ksa_paged_read(pages.cache, cu, start, n)
        here = torch.from_numpy(~gone).cuda()
        assert torch.equal(k2[here].double(), stands_for(k, fp8)[here]) and torch.equal(v2[here].double(), stands_for(v, fp8)[here])
        assert bool(torch.isnan(k2[~here].float()).all()) and bool(torch.isnan(v2[~here].float()).all())
        for rows, n_splits in ((1, 1), (5, 2), (100, 1), (100, 2)):
            for first in (n - rows, 18 * 16 + 3, 40):
                count = min(rows, n - first)
                cu, start = batch_of([first], [count])
                q = randn(count, 2, 64, seed=9)
                o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, n_splits=n_splits)
                sees = torch.from_numpy((mask(np.arange(first, first + count), n, 16, 2, 1) & gone).any(1)).cuda()
                want, _, off, _ = attend(q.double(), stands_for(k, fp8), stands_for(v, fp8), list(range(first, first + count)), p)
                assert bool(torch.isnan(o[sees].float()).all()) and bool(torch.isnan(lse[sees]).all())
                assert bool(((o.double() - want).abs() <= off)[~sees].all())


@pytest.mark.parametrize("rows,n_splits", [(5, 1), (5, 2), (100, 1), (100, 2)])
def test_exponents_at_the_front_of_the_pool_do_not_reach_rows_by_missing_pages(rows, n_splits):
    """A missing page's keys, unseen by some of the rows: whatever is read in their place is any number times any power of two."""
    say(f"paged missing pages, wild exponents rows={rows} splits={n_splits}")
    p = K.make_params(1, 1024, 16, 2, 1, 2, 1, 64)
    n = 18 * 20
    pages = Pages(p, [n], 8, True, 5, fill=448.0)
    used = torch.cat([pages.text.flatten(), pages.sums.flatten()]).tolist()
    unused = next(x for x in range(1, pages.k.shape[0]) if x not in used)
    for host, dev in ((pages.text, pages.text_dev), (pages.sums, pages.sums_dev)):
        host[host == 0] = unused
        dev.copy_(host)
    pages.k_exp.fill_(255), pages.v_exp.fill_(255)
    k, v = randn(n, 1, 64, seed=6), randn(n, 1, 64, seed=7)
    pages.put(0, 0, k, v)
    from tests.paged import kinds, mask
    _, text, idx = kinds(n, 16, 2)
    gone = text & (idx // 8 == 33)                       # rows 264 .. 271, the back half of chunk 16
    pages.text_dev[0, 33] = -1
    for first in (18 * 16 + 8, 18 * 17 + 14):            # the first rows see them, with the second start the last ones do not
        count = min(rows, n - first)
        q = randn(count, 2, 64, seed=9)
        o, lse = K.ksa_paged_fwd(pages.cache, q, *batch_of([first], [count]), n_splits=n_splits)
        sees = torch.from_numpy((mask(np.arange(first, first + count), n, 16, 2, 1) & gone).any(1)).cuda()
        want, want_lse, off, lse_off = attend(q.double(), stands_for(k, True), stands_for(v, True), list(range(first, first + count)), p)
        assert bool(torch.isnan(o[sees].float()).all()) and bool(torch.isnan(lse[sees]).all())
        assert bool(((o.double() - want).abs() <= off)[~sees].all()) and bool(((lse.double() - want_lse).abs() <= lse_off)[~sees].all())


def test_narrow_tables_are_tables_of_missing_pages():
    p = K.make_params(1, 1024, 16, 2, 1, 2, 1, 64)
    pages = Pages(p, [100], 8, False, 5)
    narrow = K.PagedCache(p, pages.k, pages.v, pages.text_dev[:, :3].contiguous(), pages.sums_dev[:, :1].contiguous())
    k = randn(100, 1, 64, seed=1)
    cu, start = batch_of([0], [100])
    K.ksa_paged_append(narrow, k, k, cu, start)
    k2, _ = K.ksa_paged_read(narrow, cu, start, 100)
    from tests.paged import kinds
    _, text, idx = kinds(100, 16, 2)
    here = torch.from_numpy(np.where(text, idx < 24, idx < 8)).cuda()
    assert torch.equal(bits(k2[here]), bits(k[here])) and bool(torch.isnan(k2[~here].float()).all())
    o, lse = K.ksa_paged_fwd(narrow, randn(1, 2, 64, seed=2), *batch_of([99], [1]))
    assert bool(torch.isnan(o.float()).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("rows", [1, 70])
@pytest.mark.parametrize("n_splits", [1, 2])
def test_sequences_out_of_place(rows, n_splits):
    """Negative or too large starts, too many rows: NaN for those sequences (nothing written by append), the others as ever; rows of no
    sequence stay as they are."""
    say(f"paged out of place rows={rows} splits={n_splits}")
    p = K.make_params(4, 256, 16, 2, 1, 4, 2, 64)
    L = 288
    pages = Pages(p, [L] * 4, 16, False, 5, fill=1.0)
    seqs = [(randn(L, 2, 64, seed=b), randn(L, 2, 64, seed=10 + b)) for b in range(4)]
    for b, (k, v) in enumerate(seqs):
        pages.put(b, 0, k, v)
    lead, total = 3, 4 * rows + 3 + 6
    cu = torch.arange(lead, lead + 4 * rows + 1, rows, dtype=torch.int32, device="cuda")
    start = torch.tensor([-1, 100, L - rows + 1, L - rows], dtype=torch.int32, device="cuda")
    q = randn(total, 4, 64, seed=20)
    o, lse = torch.full_like(q, 7.0), torch.full((total, 4), 7.0, device="cuda")
    K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, o=o, lse=lse, n_splits=n_splits)
    at = [slice(lead + b * rows, lead + (b + 1) * rows) for b in range(4)]
    for b in (0, 2):
        assert bool(torch.isnan(o[at[b]].float()).all()) and bool(torch.isnan(lse[at[b]]).all())
    for b, a0 in ((1, 100), (3, L - rows)):
        want, _, off, _ = attend(q[at[b]].double(), seqs[b][0].double(), seqs[b][1].double(), list(range(a0, a0 + rows)), p)
        assert bool(((o[at[b]].double() - want).abs() <= off).all())
    for x, y in ((o, 7.0), (lse, 7.0)):
        assert bool((x[:lead] == y).all()) and bool((x[lead + 4 * rows:] == y).all())
    before = pages.k.clone()
    kv = randn(total, 2, 64, seed=21)
    only_bad = torch.tensor([-5, L, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    K.ksa_paged_append(pages.cache, kv, kv, cu, only_bad)
    assert torch.equal(bits(pages.k), bits(before))
    k2, _ = K.ksa_paged_read(pages.cache, cu, only_bad, total)
    assert bool(torch.isnan(k2[lead:lead + 4 * rows].float()).all())
    # more rows than the call was sized for
    if rows > 1:
        K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows - 1, o=o, lse=lse, n_splits=n_splits)
        assert bool(torch.isnan(o[lead:lead + 4 * rows].float()).all()) and bool((o[lead + 4 * rows:] == 7.0).all())
    # entries of cu_rows outside the tensors
    wild = torch.tensor([-4, rows, rows, total, total + 9], dtype=torch.int32, device="cuda")
    o.fill_(7.0)
    K.ksa_paged_fwd(pages.cache, q, wild, torch.zeros_like(start) + 5, o=o, lse=lse, n_splits=n_splits)
    assert bool(torch.isnan(o[:rows].float()).all())


def test_many_sequences():
    """More than 64 sequences, some without rows."""
    B = 150
    p = K.make_params(B, 512, 16, 2, 1, 4, 2, 64)
    count = [0 if b % 7 == 3 else 1 + b % 3 for b in range(B)]
    first = [(37 * b) % 400 for b in range(B)]
    say("paged many sequences")
    check_attention(p, 16, False, first, count, 30, 1, 3)
    check_attention(p, 16, False, first, count, 30, 2, 40)
    pages = Pages(p, [a + n for a, n in zip(first, count)], 16, True, 1)
    k = randn(sum(count), 2, 64, seed=3)
    cu, start = batch_of(first, count)
    K.ksa_paged_append(pages.cache, k, k, cu, start)
    k2, v2 = K.ksa_paged_read(pages.cache, cu, start, sum(count))
    assert torch.equal(k2.double(), stands_for(k, True)) and torch.equal(k2, v2)


def test_pages_further_apart_than_32_bits():
    """A pool of 9 GB of which a sequence uses the first and the last pages."""
    say("paged far pages")
    p = K.make_params(1, 4096, 64, 8, 1, 4, 1, 128)
    n_pages, page = 36000, 1024
    pool = torch.empty(n_pages, 1, page, 128, dtype=torch.bfloat16, device="cuda")
    other = torch.empty(n_pages, 1, page, 128, dtype=torch.bfloat16, device="cuda")
    text = torch.tensor([[n_pages - 1, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    sums = torch.tensor([[n_pages - 3]], dtype=torch.int32, device="cuda")
    cache = K.PagedCache(p, pool, other, text, sums)
    n = 3000
    k, v = randn(n, 1, 128, seed=1), randn(n, 1, 128, seed=2)
    cu, start = batch_of([0], [n])
    K.ksa_paged_append(cache, k, v, cu, start)
    k2, v2 = K.ksa_paged_read(cache, cu, start, n)
    assert torch.equal(bits(k2), bits(k)) and torch.equal(bits(v2), bits(v))
    for rows in (1, 100):
        q = randn(rows, 4, 128, seed=3)
        o, _ = K.ksa_paged_fwd(cache, q, *batch_of([n - rows], [rows]))
        want, _, off, _ = attend(q.double(), k.double(), v.double(), list(range(n - rows, n)), p)
        assert bool(((o.double() - want).abs() <= off).all())


# ---- together, as they are used -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
def test_a_prompt_in_pieces_then_tokens(fp8):
    """Two prompts in pieces of any size, then single rows and drafted ones: every row's output is that of the whole sequence."""
    say(f"paged generate fp8={fp8}")
    p = K.make_params(2, 1024, 16, 2, 2, 8, 2, 128)
    L = [500, 333]
    pages = Pages(p, L, 16, fp8, 5)
    k, v = [randn(n, 2, 128, seed=b) for b, n in enumerate(L)], [randn(n, 2, 128, seed=5 + b) for b, n in enumerate(L)]
    q = [randn(n, 8, 128, seed=10 + b) for b, n in enumerate(L)]
    done, outs = [0, 0], [[], []]
    pieces = [(200, 33), (7, 100), (150, 64), (1, 1), (5, 3), (1, 0), (0, 1), (100, 90)]
    while done != L:
        count = [min(x, n - d) for x, n, d in zip(pieces[0], L, done)]
        pieces = pieces[1:] + pieces[:1]
        cu, start = batch_of(done, count)
        take = lambda x: torch.cat([x[b][done[b]:done[b] + count[b]] for b in range(2)])  # noqa: E731
        K.ksa_paged_append(pages.cache, take(k), take(v), cu, start)
        o, _ = K.ksa_paged_fwd(pages.cache, take(q), cu, start, max_rows=max(max(count), 1))
        outs[0].append(o[:count[0]]), outs[1].append(o[count[0]:])
        done = [d + n for d, n in zip(done, count)]
    for b in range(2):
        o = torch.cat(outs[b]).double()
        want, _, off, _ = attend(q[b].double(), stands_for(k[b], fp8), stands_for(v[b], fp8), list(range(L[b])), p)
        assert bool(((o - want).abs() <= off).all()), float(((o - want).abs() / off).max())


def test_the_whole_sequence_agrees_with_prefill_and_decode():
    """A prompt by ksa_prefill_fwd, its k and v into the pages, and the next token by ksa_decode_fwd over the ring cache: the same outputs."""
    say("paged against prefill and decode")
    B, Hq, Hkv, d, c, m, C, n = 2, 8, 2, 128, 64, 8, 1, 700
    p = K.make_params(B, n, c, m, C, Hq, Hkv, d)
    L = n // c * (c + m) + n % c
    q, k, v = randn(B * L, Hq, d, seed=1), randn(B * L, Hkv, d, seed=2), randn(B * L, Hkv, d, seed=3)
    o, lse = K.ksa_prefill_fwd(K.ksa_build_layout(p), q.view(B, L, Hq, d), k.view(B, L, Hkv, d), v.view(B, L, Hkv, d))
    pages = Pages(p, [L] * B, 32, False, 4)
    cu, start = batch_of([0] * B, [L] * B)
    K.ksa_paged_append(pages.cache, k, v, cu, start)
    o2, lse2 = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=L)
    # either is off by half a step of its output and of every weight; prefill's log-sum-exp may come from rounded weights
    bar = 4 * 2.0 ** -8 * float(v.abs().max())
    assert float((o2.double() - o.view(B * L, Hq, d).double()).abs().max()) < bar
    _, _, _, off = attend(q[:L].double(), k[:L].double(), v[:L].double(), list(range(L)), p)
    assert float((lse2.view(B, L, Hq).permute(0, 2, 1).double() - lse.double()).abs().max()) < 2.0 ** -8 + 2 * float(off.max())
    last = [L - 1] * B
    at = torch.tensor([L - 1, 2 * L - 1], device="cuda")
    k_cache = torch.zeros(B, Hkv, K.cache_geometry(p)[1], d, dtype=torch.bfloat16, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    K.ksa_cache_from_prefill(p, n, k.view(B, L, Hkv, d), v.view(B, L, Hkv, d), k_cache, v_cache)
    od, lsed = K.ksa_decode_fwd(p, q[at].contiguous(), k_cache, v_cache, torch.full((B,), n - 1, dtype=torch.int32, device="cuda"))
    o1, lse1 = K.ksa_paged_fwd(pages.cache, q[at].contiguous(), *batch_of(last, [1] * B), max_rows=1)
    assert float((o1.double() - od.double()).abs().max()) < bar and float((lse1 - lsed).abs().max()) < 2 * float(off.max())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows,n_splits", [(1, 4), (1, 1), (40, 3)])
def test_graph_replays_with_new_rows_tables_and_places(rows, n_splits, fp8):
    """Append and attention captured once; between replays the rows, starts, the batch's borders and a table change."""
    say(f"paged graph rows={rows} splits={n_splits} fp8={fp8}")
    B = 3
    p = K.make_params(B, 1024, 16, 2, 2, 8, 2, 64)
    L = [400, 300, 350]
    pages = Pages(p, L, 16, fp8, 5)
    spare = Pages(p, L, 16, fp8, 5)
    total = B * rows
    q, k, v = (torch.empty(total, h, 64, dtype=torch.bfloat16, device="cuda") for h in (8, 2, 2))
    cu, start = batch_of([0] * B, [rows] * B)
    o, lse = torch.zeros_like(q), torch.zeros(total, 8, device="cuda")
    ws = [torch.empty(max(K.paged_workspace_bytes(pages.cache, total, rows, n_splits), 16), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(cache, o, lse, ws):
        K.ksa_paged_append(cache, k, v, cu, start)
        K.ksa_paged_fwd(cache, q, cu, start, max_rows=rows, o=o, lse=lse, workspace=ws, n_splits=n_splits)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(pages.cache, o, lse, ws[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pages.cache, o, lse, ws[0])
    for turn in range(4):
        for b in range(B):
            pages.put(b, 0, randn(L[b], 2, 64, seed=100 * turn + b), randn(L[b], 2, 64, seed=100 * turn + 50 + b))
        if turn == 2:      # two pages change places
            for t in (pages.text_dev, pages.text):
                t[:, [0, 1]] = t[:, [1, 0]].clone()
        for x in ("k", "v", "k_exp", "v_exp"):
            if getattr(pages, x) is not None:
                getattr(spare, x).copy_(getattr(pages, x))
        spare.text_dev.copy_(pages.text_dev)
        q.copy_(randn(total, 8, 64, seed=turn)), k.copy_(randn(total, 2, 64, seed=turn + 20)), v.copy_(randn(total, 2, 64, seed=turn + 40))
        start.copy_(torch.tensor([L[b] - rows - 11 * turn - b for b in range(B)], dtype=torch.int32))
        if turn == 3:
            cu.copy_(torch.tensor([0, rows, rows, 2 * rows], dtype=torch.int32))      # one sequence has none
        o.fill_(7.0), lse.fill_(7.0)
        o2, lse2 = o.clone(), lse.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(spare.cache, o2, lse2, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(bits(o), bits(o2)) and torch.equal(lse, lse2)
        assert torch.equal(pages.k.view(torch.uint8), spare.k.view(torch.uint8))


def test_a_stream_of_its_own_and_repeated_calls():
    say("paged streams")
    p = K.make_params(2, 2048, 64, 8, 1, 8, 2, 128)
    pages = Pages(p, [1500, 900], 64, False, 5)
    for b, n in enumerate((1500, 900)):
        pages.put(b, 0, randn(n, 2, 128, seed=b), randn(n, 2, 128, seed=b + 5))
    for rows in (1, 64):
        q = randn(2 * rows, 8, 128, seed=3)
        cu, start = batch_of([1500 - rows, 900 - rows], [rows, rows])
        o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=4)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        outs = [K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=4, stream=s, o=torch.empty_like(q), lse=torch.empty_like(lse0),
                                workspace=torch.empty(K.paged_workspace_bytes(pages.cache, 2 * rows, rows, 4), dtype=torch.uint8, device="cuda"))
                for s in streams]
        torch.cuda.synchronize()
        for o, lse in outs:
            assert torch.equal(bits(o), bits(o0)) and torch.equal(lse, lse0)


@pytest.mark.parametrize("rows", [1, 64])
def test_what_a_call_allocates_belongs_to_its_stream(rows):
    """Outputs and workspaces of calls on another stream, whose memory is given back and taken again while they run."""
    say(f"paged allocations rows={rows}")
    p = K.make_params(2, 8192, 64, 8, 1, 8, 2, 128)
    pages = Pages(p, [9000, 8000], 64, False, 5)
    for b, n in enumerate((9000, 8000)):
        pages.put(b, 0, randn(n, 2, 128, seed=b), randn(n, 2, 128, seed=b + 5))
    q = randn(2 * rows, 8, 128, seed=3)
    cu, start = batch_of([9000 - rows, 8000 - rows], [rows, rows])
    o0, lse0 = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=4)
    k0, v0 = K.ksa_paged_read(pages.cache, cu, start, 2 * rows)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    size = K.paged_workspace_bytes(pages.cache, 2 * rows, rows, 4)
    for _ in range(8):
        o, lse = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=4, stream=side)
        torch.full((size,), 255, dtype=torch.uint8, device="cuda")        # on the current stream, at once
        k, v = K.ksa_paged_read(pages.cache, cu, start, 2 * rows, stream=side)
        torch.full_like(k, 9.0)
        torch.cuda.synchronize()
        assert torch.equal(bits(o), bits(o0)) and torch.equal(lse, lse0) and torch.equal(bits(k), bits(k0)) and torch.equal(bits(v), bits(v0))


def test_two_graphs_share_a_workspace():
    say("paged graphs, one workspace")
    p = K.make_params(2, 4096, 64, 8, 1, 8, 2, 128)
    pages = Pages(p, [3000, 2000], 64, True, 5)
    for b, n in enumerate((3000, 2000)):
        pages.put(b, 0, randn(n, 2, 128, seed=b), randn(n, 2, 128, seed=b + 5))
    calls, graphs = [], []
    ws = torch.empty(max(K.paged_workspace_bytes(pages.cache, 2 * rows, rows, 4) for rows in (1, 64)), dtype=torch.uint8, device="cuda")
    for rows in (1, 64):
        q = randn(2 * rows, 8, 128, seed=3)
        cu, start = batch_of([3000 - rows, 2000 - rows], [rows, rows])
        want = K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=4)
        got = torch.empty_like(want[0]), torch.empty_like(want[1])
        calls.append((q, cu, start, want, got))
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            K.ksa_paged_fwd(pages.cache, q, cu, start, max_rows=rows, n_splits=4, workspace=ws, o=got[0], lse=got[1])
        graphs.append(g)
    for turn in range(4):
        for _, _, _, _, got in calls:
            got[0].zero_(), got[1].zero_()
        ws.fill_(255)                                      # (NaN)
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for _, _, _, want, got in calls:
            assert torch.equal(bits(want[0]), bits(got[0])) and torch.equal(want[1], got[1])


def test_a_cache_keeps_its_own_parameters():
    p = K.make_params(1, 1024, 16, 2, 1, 2, 1, 64)
    pages = Pages(p, [100], 8, False, 5)
    p.batch, p.n_kv_heads = 50, 2
    k = randn(100, 1, 64, seed=1)
    cu, start = batch_of([0], [100])
    K.ksa_paged_append(pages.cache, k, k, cu, start)
    k2, _ = K.ksa_paged_read(pages.cache, cu, start, 100)
    assert torch.equal(bits(k2), bits(k))


def test_python_refuses_what_does_not_fit():
    p = K.make_params(2, 1024, 16, 2, 1, 4, 2, 64)
    pages = Pages(p, [100, 50], 8, True, 5)
    c = pages.cache
    half = torch.zeros(10, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(10, 4, 64, dtype=torch.bfloat16, device="cuda")
    cu, start = batch_of([0, 0], [6, 4])
    k, v, t, u, ke, ve = pages.k, pages.v, pages.text_dev, pages.sums_dev, pages.k_exp, pages.v_exp
    for make in (lambda: K.PagedCache(p, k, v, t, u), lambda: K.PagedCache(p, k, v, t, u, ke), lambda: K.PagedCache(p, k, v, t, None, ke, ve),
                 lambda: K.PagedCache(p, k.float(), v.float(), t, u), lambda: K.PagedCache(p, k, v[1:], t, u, ke, ve),
                 lambda: K.PagedCache(p, k, v.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3), t, u, ke, ve),
                 lambda: K.PagedCache(p, k, v, t[:1], u, ke, ve), lambda: K.PagedCache(p, k, v, t.long(), u, ke, ve),
                 lambda: K.PagedCache(p, k, v, t[:, ::2], u, ke, ve), lambda: K.PagedCache(p, k, v, t.cpu(), u, ke, ve),
                 lambda: K.PagedCache(p, k, v, t, u, ke[1:], ve), lambda: K.PagedCache(p, k.cpu(), v, t, u, ke, ve)):
        with pytest.raises(ValueError):
            make()
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for call in (lambda: K.ksa_paged_append(c, half.float(), half, cu, start), lambda: K.ksa_paged_append(c, half[:, :1], half[:, :1], cu, start),
                 lambda: K.ksa_paged_append(c, half, half[:9], cu, start), lambda: K.ksa_paged_append(c, half, half, cu[:2], start),
                 lambda: K.ksa_paged_append(c, half, half, cu, start.long()), lambda: K.ksa_paged_append(c, half, half, cu.cpu(), start),
                 lambda: K.ksa_paged_append(c, half, half.cpu(), cu, start), lambda: K.ksa_paged_append(c, half, q[:, ::2], cu, start),
                 lambda: K.ksa_paged_read(c, cu, start, 9, k=half), lambda: K.ksa_paged_read(c, cu, start, 10, k=half, v=q[:, ::2]),
                 lambda: K.ksa_paged_fwd(c, half, cu, start), lambda: K.ksa_paged_fwd(c, q[..., ::2], cu, start),
                 lambda: K.ksa_paged_fwd(c, q, cu, start, o=q.float()), lambda: K.ksa_paged_fwd(c, q, cu, start, lse=torch.zeros(4, 10, device="cuda")),
                 lambda: K.ksa_paged_fwd(c, q, cu, start, workspace=ws.float()), lambda: K.ksa_paged_fwd(c, q, cu, start, workspace=ws.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: K.ksa_paged_fwd(c, q, cu, start, n_splits=-1), lambda: K.ksa_paged_fwd(c, q, cu, start, max_rows=0),
                 lambda: K.ksa_paged_fwd(c, q, cu, start, n_splits=2, workspace=ws[:16]), lambda: K.ksa_paged_fwd(c, q, cu, start, n_splits=2, workspace=ws[1:]),
                 lambda: K.ksa_paged_fwd(c, torch.cat([q, q]).as_strided((10, 4, 64), (260, 64, 1)), cu, start, o=torch.empty_like(q))):
        with pytest.raises(K.KsaError):
            call()
