"""GPU tests of rotary positions: whole sequences, there and back, and a serving step's rows, against definitions in 64 bits (tests/rotary.py)."""
import math

import numpy as np
import pytest
import torch

import paper_2604_24432_amd as K
from tests.paged import Pages, batch_of, randn
from tests.paged_fp4 import Pages4
from tests.rotary import RULES, handle, name, positions, turn
from tests.test_gpu_paged import bits, say

pytestmark = pytest.mark.gpu


def within(got, x, rule, at, back=False):
    want, off = turn(x.double(), rule, at, back)
    err = (got.double() - want).abs()
    assert bool((err <= off).all()), float((err - off).max())


# batch, heads, KV heads, d, text tokens, c, m
SHAPES = [(1, 1, 1, 128, 1, 64, 8), (2, 4, 2, 128, 150, 64, 8), (1, 12, 4, 64, 333, 48, 6), (3, 5, 1, 128, 40, 1, 0), (1, 32, 8, 128, 1000, 8, 1), (1, 33, 3, 64, 20, 100, 4)]


@pytest.mark.parametrize("rule", RULES, ids=name)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_whole_sequences(shape, rule):
    B, Hq, Hkv, d, n, c, m = shape
    rule = {**rule, "dim": min(rule["dim"], d)}
    say(f"rotary whole {shape} {rule}")
    p = K.make_params(B, n, c, m, 1, Hq, Hkv, d)
    L = K.binding.augmented_rows(p, n)
    at = positions(range(L), c, m)
    assert at.tolist() == K.Layout(p).index_maps()["position_ids"].tolist()
    r = handle(rule)
    q, k = randn(B, L, Hq, d, seed=1), randn(B, L, Hkv, d, seed=2)
    for back, call in ((False, K.ksa_rotary_fwd), (True, K.ksa_rotary_bwd)):
        q0, k0 = q.clone(), k.clone()
        q_out, k_out = call(p, r, q0, k0)
        assert torch.equal(bits(q0), bits(q)) and torch.equal(bits(k0), bits(k))
        within(q_out, q, rule, at, back), within(k_out, k, rule, at, back)
        only_q, none = call(p, r, q, None)
        none_, only_k = call(p, r, None, k)
        assert none is None and none_ is None and torch.equal(bits(only_q), bits(q_out)) and torch.equal(bits(only_k), bits(k_out))
        call(p, r, q0, k0, q0, k0)                       # in place
        assert torch.equal(bits(q0), bits(q_out)) and torch.equal(bits(k0), bits(k_out))


def test_strides_of_a_fused_projection():
    say("rotary strides")
    p = K.make_params(2, 100, 16, 2, 1, 4, 2, 128)
    L = K.binding.augmented_rows(p, 100)
    rule = RULES[3]
    fused = randn(2, L, 9, 128, seed=1)
    before = fused.clone()
    q, k = fused[:, :, :4], fused[:, :, 4:6]
    out = torch.full((2, 9, L, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    K.ksa_rotary_fwd(p, handle(rule), q, k, out[:, :4].transpose(1, 2), out[:, 5:7].transpose(1, 2))
    at = positions(range(L), 16, 2)
    within(out[:, :4].transpose(1, 2), q, rule, at), within(out[:, 5:7].transpose(1, 2), k, rule, at)
    assert bool((out[:, 4] == 7).all()) and bool((out[:, 7:] == 7).all()) and torch.equal(bits(fused), bits(before))
    K.ksa_rotary_fwd(p, handle(rule), q, k, q, k)
    within(fused[:, :, :4], before[:, :, :4], rule, at), within(fused[:, :, 4:6], before[:, :, 4:6], rule, at)
    assert torch.equal(bits(fused[:, :, 6:]), bits(before[:, :, 6:]))


@pytest.mark.parametrize("rule", [RULES[0], RULES[3], RULES[4]], ids=name)
def test_gradients_against_differences(rule):
    """Linear in its input: <g, R (x + h e) - R x> / h is the gradient, to the roundings of both (float64 sums of the kernels' outputs)."""
    say("rotary differences")
    p = K.make_params(1, 50, 16, 2, 1, 2, 1, 128)
    L = K.binding.augmented_rows(p, 50)
    r = handle(rule)
    g = randn(1, L, 2, 128, seed=3)
    dq, _ = K.ksa_rotary_bwd(p, r, g, None)
    zero, _ = K.ksa_rotary_fwd(p, r, torch.zeros_like(g), None)
    assert bool((zero == 0).all())
    picks = [(0, 0, 0), (17, 1, 5), (31, 0, 64), (L - 1, 1, 127), (40, 0, 9), (12, 1, 70)]
    for row, head, e in picks:
        x = torch.zeros_like(g)
        x[0, row, head, e] = 1.0
        y, _ = K.ksa_rotary_fwd(p, r, x, None)
        diff = float((g.double() * y.double()).sum())
        # the difference has two outputs, each off by half a step of bf16, the gradient has one such step
        size = float((g.double() * y.double()).abs().sum())
        assert abs(float(dq[0, row, head, e]) - diff) <= 2 ** -8 * (size + abs(diff)) + 2.0 ** -19 * float(g[0, row, head].abs().max()), (row, head, e)


def test_no_numbers_stay_in_their_pairs():
    say("rotary no numbers")
    p = K.make_params(1, 30, 16, 2, 1, 2, 1, 64)
    L = K.binding.augmented_rows(p, 30)
    q = randn(1, L, 2, 64, seed=1)
    for rule in (dict(dim=32), dict(dim=32, interleaved=True), dict(dim=20), dict(dim=22, interleaved=True)):
        r = handle(rule)
        y0, _ = K.ksa_rotary_fwd(p, r, q, None)
        for e in (0, 5, rule["dim"] - 1, rule["dim"], 63):
            x = q.clone()
            x[0, 7, 1, e] = math.nan
            y, _ = K.ksa_rotary_fwd(p, r, x, None)
            hit = torch.zeros_like(y, dtype=torch.bool)
            half = rule["dim"] // 2
            pair = [e] if e >= rule["dim"] else [e, e ^ 1] if rule.get("interleaved") else [e, (e + half) % rule["dim"]]
            hit[0, 7, 1, pair] = True
            assert bool(torch.isnan(y[hit]).all()) and torch.equal(bits(y)[~hit], bits(y0)[~hit]), (rule, e)


def test_far_positions():
    """Rows of whole sequences near the end of a million positions, through the paged form too."""
    say("rotary far")
    n, c, m = 1 << 20, 64, 8
    p = K.make_params(1, n, c, m, 1, 1, 1, 64)
    L = K.binding.augmented_rows(p, n)
    rows = np.concatenate([np.arange(5), np.arange(L // 3, L // 3 + 100), np.arange(L - 300, L)])
    for rule in (dict(dim=64), dict(dim=64, base=1e6, interleaved=True), dict(dim=20, scaling="linear", factor=3.0)):
        q = randn(1, L, 1, 64, seed=1)
        out, _ = K.ksa_rotary_fwd(p, handle(rule), q, None)
        within(out[:, rows], q[:, rows], rule, positions(rows, c, m))


def make(p, n_rows, page, kind, seed):
    return Pages4(p, n_rows, page, seed) if kind == "fp4" else Pages(p, n_rows, page, kind == "fp8", seed, fill=0.0)


PLACES = [(1, 8, 1, 64, 8, 1, 16, [786], [1]), (6, 32, 8, 128, 64, 8, 64, [0, 1, 63, 64, 71, 72], [1] * 6), (4, 12, 4, 64, 48, 6, 8, [1500, 53, 160, 7], [77, 0, 301, 1]),
          (2, 5, 5, 128, 1, 0, 16, [40, 3], [33, 90])]


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("rule", [RULES[0], RULES[1], RULES[3], RULES[4], RULES[6]], ids=name)
@pytest.mark.parametrize("case", PLACES, ids=lambda x: "x".join(map(str, x[:7])))
def test_new_rows_into_pages(case, rule, kind):
    """The same bits as turning (ksa_rotary_fwd's, by position) and ksa_paged_append; q to its bound."""
    B, Hq, Hkv, d, c, m, page, first, count = case
    rule = {**rule, "dim": min(rule["dim"], d)}
    say(f"rotary place {case} {rule} {kind}")
    p = K.make_params(B, 4096, c, m, 1, Hq, Hkv, d)
    r = handle(rule)
    total = sum(count)
    q, k, v = randn(total + 2, Hq, d, seed=1), randn(total + 2, Hkv, d, seed=2), randn(total + 2, Hkv, d, seed=3)
    cu, start = batch_of(first, count)
    n_rows = [a + n for a, n in zip(first, count)]
    got, want = make(p, n_rows, page, kind, 5), make(p, n_rows, page, kind, 5)
    q_out = torch.full_like(q, 7.0)
    K.ksa_paged_rotary(got.cache, r, q, k, v, cu, start, q_out=q_out)
    assert bool((q_out[total:] == 7).all())
    # k turned by the call for whole sequences, every row at its place
    whole = K.make_params(1, 4096, c, m, 1, Hkv, Hkv, d)
    L = K.binding.augmented_rows(whole, 4096)
    at, k_turned = 0, k.clone()
    for b, n in enumerate(count):
        rows = list(range(first[b], first[b] + n))
        within(q_out[at:at + n], q[at:at + n], rule, positions(rows, c, m))
        line = torch.zeros(1, L, Hkv, d, dtype=torch.bfloat16, device="cuda")
        line[0, rows] = k[at:at + n]
        k_turned[at:at + n] = K.ksa_rotary_fwd(whole, r, None, line)[1][0, rows]
        at += n
    K.ksa_paged_append(want.cache, k_turned, v, cu, start)
    for x in ("k", "v", "k_exp", "v_exp"):
        a, b = getattr(got, x), getattr(want, x)
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)), x
    # in place, without q, and strided
    again = make(p, n_rows, page, kind, 5)
    assert K.ksa_paged_rotary(again.cache, r, None, k, v, cu, start) is None
    assert torch.equal(again.k.view(torch.uint8), got.k.view(torch.uint8))
    fused = torch.cat([q, k, v], 1)
    strided = make(p, n_rows, page, kind, 5)
    K.ksa_paged_rotary(strided.cache, r, fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:], cu, start, q_out=fused[:, :Hq])
    assert torch.equal(bits(fused[:total, :Hq]), bits(q_out[:total])) and torch.equal(bits(fused[total:, :Hq]), bits(q[total:]))
    assert torch.equal(strided.k.view(torch.uint8), got.k.view(torch.uint8)) and torch.equal(strided.v.view(torch.uint8), got.v.view(torch.uint8))


def test_sequences_out_of_place_and_rows_without_a_page():
    say("rotary out of place")
    p = K.make_params(3, 500, 16, 2, 1, 4, 2, 64)
    r = handle(dict(dim=64))
    q, k, v = randn(30, 4, 64, seed=1), randn(30, 2, 64, seed=2), randn(30, 2, 64, seed=3)
    pages = Pages(p, [200, 200, 200], 16, False, 5, fill=0.0)
    cu, start = batch_of([100, -1, 10 ** 6], [10, 10, 10])
    q_out = K.ksa_paged_rotary(pages.cache, r, q, k, v, cu, start)
    within(q_out[:10], q[:10], dict(dim=64), positions(range(100, 110), 16, 2))
    assert bool(torch.isnan(q_out[10:]).all())
    assert int((pages.k != 0).any(-1).any(1).sum()) == 10
    none = torch.full_like(pages.text_dev, -1)
    empty = K.PagedCache(p, torch.zeros_like(pages.k), torch.zeros_like(pages.v), none, torch.full_like(pages.sums_dev, -1))
    q_out = K.ksa_paged_rotary(empty, r, q, k, v, *batch_of([100, 50, 0], [10, 10, 10]))
    assert bool(torch.isfinite(q_out).all()) and not bool(empty.k.any())
    assert K.ksa_paged_rotary(empty, r, q[:0], k[:0], v[:0], *batch_of([0, 0, 0], [0, 0, 0])).shape[0] == 0


def test_graph_and_streams():
    """Captured with a training step's eager calls beside it; replays with new data give the eager bits."""
    say("rotary graph")
    p = K.make_params(1, 200, 16, 2, 1, 4, 2, 128)
    L = K.binding.augmented_rows(p, 200)
    r = handle(RULES[0])
    q, k = randn(1, L, 4, 128, seed=1), randn(1, L, 2, 128, seed=2)
    q_out, k_out, dq, dk = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k)
    pages = Pages(p, [L], 16, False, 5, fill=0.0)
    cu, start = batch_of([0], [9])

    def step():
        K.ksa_rotary_fwd(p, r, q, k, q_out, k_out)
        K.ksa_rotary_bwd(p, r, q_out, k_out, dq, dk)
        K.ksa_paged_rotary(pages.cache, r, q[0, :9], k[0, :9], k[0, :9], cu, start, q_out=q_out[0, :9])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x in range(4):
        q.copy_(randn(1, L, 4, 128, seed=10 + x)), k.copy_(randn(1, L, 2, 128, seed=20 + x))
        start.fill_(7 * x)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q_out, k_out, dq, dk, pages.k)]
        pages.k.zero_()
        step()
        pages_k = pages.k.clone()
        for a, b in zip(got[:4], (q_out, k_out, dq, dk)):
            assert torch.equal(bits(a), bits(b))
        written = (pages_k != 0).any(-1)
        assert torch.equal(bits(got[4][written]), bits(pages_k[written]))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    a, b = K.ksa_rotary_fwd(p, r, q, k, stream=stream)
    c = K.ksa_paged_rotary(pages.cache, r, q[0, :9], k[0, :9], k[0, :9], cu, start, stream=stream)
    stream.synchronize()
    want = K.ksa_rotary_fwd(p, r, q, k)
    assert torch.equal(bits(a), bits(want[0])) and torch.equal(bits(b), bits(want[1])) and bool(torch.isfinite(c).all())


def test_python_refuses_what_does_not_fit():
    p = K.make_params(1, 100, 16, 2, 1, 4, 2, 128)
    L = K.binding.augmented_rows(p, 100)
    r = handle(RULES[0])
    q, k = randn(1, L, 4, 128), randn(1, L, 2, 128)
    for bad in ((q[:, 1:], k), (q, q), (q.float(), k), (None, None), (q, k[..., :64]), (q.cpu(), k), (q, k, q[:, :1]), (q, None, None, k)):
        with pytest.raises(ValueError):
            K.ksa_rotary_fwd(p, r, *bad)
    with pytest.raises(K.KsaError):
        K.ksa_rotary_fwd(K.make_params(1, 100, 16, 2, 1, 4, 2, 64), r, q[..., :64].contiguous(), None)      # dim beyond the head
    pages = Pages(p, [100], 16, False, 5)
    cu, start = batch_of([0], [5])
    x, y = q[0, :5], k[0, :5]
    for bad in ((x, y, y[:4], cu, start), (x[:4], y, y, cu, start), (x, y, y, cu[:1], start), (x, y, y, cu.long(), start), (None, y, y, cu, start, x), (y, y, y, cu, start)):
        with pytest.raises(ValueError):
            K.ksa_paged_rotary(pages.cache, r, *bad)


def test_rows_further_apart_than_32_bits():
    say("rotary far rows")
    p = K.make_params(2, 40, 16, 2, 1, 3, 1, 64)
    L = K.binding.augmented_rows(p, 40)
    far = torch.empty(6 << 30, dtype=torch.uint8, device="cuda").view(torch.bfloat16)          # 3 Gi elements
    row = (3 << 30) // (2 * L + 1) // 8 * 8
    q = torch.as_strided(far, (2, L, 3, 64), (L * row, row, 64, 1))
    x = randn(2, L, 3, 64, seed=1)
    q.copy_(x)
    r = handle(dict(dim=64))
    out, _ = K.ksa_rotary_fwd(p, r, q, None, torch.empty_like(x))
    at = positions(range(L), 16, 2)
    within(out, x, dict(dim=64), at)
    K.ksa_rotary_fwd(p, r, q, None, q)
    assert torch.equal(bits(q), bits(out))
    pages = Pages(p, [L, L], 16, False, 5, fill=0.0)
    q.copy_(x)
    k = torch.as_strided(far, (2 * L, 1, 64), (row, 64, 1), 192)                               # behind the heads of q
    k.copy_(x[:, :, :1].flatten(0, 1))
    cu, start = batch_of([0, 0], [L, L])
    got = K.ksa_paged_rotary(pages.cache, r, torch.as_strided(far, (2 * L, 3, 64), (row, 64, 1)), k, k, cu, start, q_out=torch.empty_like(x).view(2 * L, 3, 64))
    assert torch.equal(bits(got.view_as(out)), bits(out))
    kb, vb = K.ksa_paged_read(pages.cache, cu, start, 2 * L)
    assert torch.equal(bits(kb.view(2, L, 1, 64)), bits(out[:, :, :1])) and torch.equal(bits(vb), bits(k.contiguous()))


def test_what_training_does_beside_captured_steps():
    """Forward, attention and backward through turned q and k: gradients of a whole layer's scores against float64 autograd of the definition."""
    say("rotary with prefill")
    p = K.make_params(1, 48, 16, 2, 1, 4, 2, 64)
    lay = K.Layout(p)
    L = lay.aug_len
    rule = dict(dim=32, base=500.0, scaling="by_parts", factor=2.0, original=64.0)
    r = handle(rule)
    q, k, v, g = (randn(1, L, h, 64, seed=s) * 0.5 for h, s in ((4, 1), (2, 2), (2, 3), (4, 4)))
    qt, kt = K.ksa_rotary_fwd(p, r, q, k)
    o, lse = K.ksa_prefill_fwd(lay, qt, kt, v)
    dqt, dkt, dv = K.ksa_prefill_bwd(lay, qt, kt, v, o, lse, g)
    dq, dk = K.ksa_rotary_bwd(p, r, dqt, dkt)
    see = torch.from_numpy(np.stack([lay.mask_row(i) for i in range(L)])).bool()
    at = positions(range(L), 16, 2)
    x = [t[0].double().cpu().requires_grad_() for t in (q, k, v)]

    def plain(y):      # the definition again, in operations that autograd can follow
        from tests.rotary import frequencies
        f, magnitude = frequencies(rule)
        angle = torch.tensor(at, dtype=torch.float64)[:, None, None] * torch.tensor(f, dtype=torch.float64)
        a, b = y[..., :16], y[..., 16:32]
        return torch.cat([(a * angle.cos() - b * angle.sin()) * magnitude, (b * angle.cos() + a * angle.sin()) * magnitude, y[..., 32:]], -1)
    qd, kd = plain(x[0]), plain(x[1])
    out = []
    for h in range(4):
        s = (qd[:, h] @ kd[:, h // 2].T / 8).masked_fill(~see, -math.inf)
        out.append(torch.softmax(s, 1) @ x[2][:, h // 2])
    torch.stack(out, 1).backward(g[0].double().cpu())
    # the bars of the prefill's own gradients (2e-2 + 2^-8 of the entry), turned: a pair's entries share theirs, times the magnitude, and one more rounding
    for got, want in ((dq, x[0].grad), (dk, x[1].grad), (dv, x[2].grad)):
        err = (got[0].double().cpu() - want).abs()
        assert bool((err <= 2 * 1.07 * 2e-2 + 2.0 ** -7 * want.abs()).all()) and float(err.mean()) <= 2 * 2e-3, float(err.max())


@pytest.mark.parametrize("rule", [dict(dim=128), dict(dim=64, interleaved=True), dict(dim=36)], ids=name)
def test_outputs_larger_than_the_caches(rule):
    """From 256 MB of output on another kernel runs: the same bits as the sequence's beginning alone, and the definition at its end; in place too."""
    say(f"rotary large {rule}")
    c, m, n = 64, 8, 60000
    p, few = K.make_params(1, n, c, m, 1, 16, 2, 128), K.make_params(1, 1000, c, m, 1, 16, 2, 128)
    L, L0 = K.binding.augmented_rows(p, n), K.binding.augmented_rows(p, 1000)
    assert L * 18 * 128 * 2 >= 256 << 20 > L0 * 18 * 128 * 2
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k = (torch.randn(1, L, h, 128, generator=g, device="cuda").to(torch.bfloat16) for h in (16, 2))
    r = handle(rule)
    for call, back in ((K.ksa_rotary_fwd, False), (K.ksa_rotary_bwd, True)):
        got = call(p, r, q, k)
        for x, y in zip(got, call(few, r, q[:, :L0].contiguous(), k[:, :L0].contiguous())):
            assert torch.equal(bits(x[:, :L0]), bits(y))
        for x, y in zip(got, (q, k)):
            within(x[:, -100:], y[:, -100:], rule, positions(range(L - 100, L), c, m), back)
    inout = q.clone()
    K.ksa_rotary_bwd(p, r, inout, None, inout)
    assert torch.equal(bits(inout), bits(got[0]))


@pytest.mark.parametrize("rule", [RULES[0], RULES[1], RULES[3], RULES[4], RULES[6]], ids=name)
@pytest.mark.parametrize("B,Hq,Hkv,d,c,m", [(1, 1, 1, 64, 16, 2), (5, 32, 8, 128, 64, 8), (300, 7, 7, 128, 8, 1), (3, 12, 4, 64, 48, 6)])
def test_single_rows_of_the_decode_loop(B, Hq, Hkv, d, c, m, rule):
    """The bits of the whole sequence's rows; sequences whose position is outside become NaN; in place, strided, q or k alone."""
    rule = {**rule, "dim": min(rule["dim"], d)}
    say(f"rotary step {B} {Hq}/{Hkv} {d} {rule}")
    n = 10 * c + c // 2
    p = K.make_params(B, n, c, m, 1, Hq, Hkv, d)
    one = K.make_params(1, n, c, m, 1, Hq, Hkv, d)
    L = K.binding.augmented_rows(p, n)
    r = handle(rule)
    q, k = randn(B, Hq, d, seed=1), randn(B, Hkv, d, seed=2)
    for kind, most in ((K.KSA_ROW_TEXT, n), (K.KSA_ROW_SUMMARY, 10 * m)):
        at = [(b * 37 + most - 1) % most for b in range(B)]
        pos = torch.tensor(at, dtype=torch.int32, device="cuda")
        q_out, k_out = K.ksa_rotary_step(p, r, kind, q, k, pos)
        rows = [x // c * (c + m) + x % c if kind == K.KSA_ROW_TEXT else x // m * (c + m) + c + x % m for x in at]
        within(q_out, q, rule, positions(rows, c, m)), within(k_out, k, rule, positions(rows, c, m))
        b = B // 2
        line = torch.zeros(1, L, Hq, d, dtype=torch.bfloat16, device="cuda")
        line[0, rows[b]] = q[b]
        assert torch.equal(bits(K.ksa_rotary_fwd(one, r, line, None)[0][0, rows[b]]), bits(q_out[b]))
        only_q, none = K.ksa_rotary_step(p, r, kind, q, None, pos)
        none_, only_k = K.ksa_rotary_step(p, r, kind, None, k, pos)
        assert none is None and none_ is None and torch.equal(bits(only_q), bits(q_out)) and torch.equal(bits(only_k), bits(k_out))
        fused = torch.cat([q, k], 1)
        K.ksa_rotary_step(p, r, kind, fused[:, :Hq], fused[:, Hq:], pos, fused[:, :Hq], fused[:, Hq:])
        assert torch.equal(bits(fused), bits(torch.cat([q_out, k_out], 1)))
        for outside in (-1, most, 2 ** 31 - 1):
            bad = pos.clone()
            bad[b] = outside
            got_q, got_k = K.ksa_rotary_step(p, r, kind, q, k, bad)
            others = torch.arange(B, device="cuda") != b
            assert bool(torch.isnan(got_q[b]).all()) and bool(torch.isnan(got_k[b]).all())
            assert torch.equal(bits(got_q[others]), bits(q_out[others])) and torch.equal(bits(got_k[others]), bits(k_out[others]))


def test_a_decode_loop_with_positions_agrees_with_the_prefill():
    """Keys turned before they are cached, queries before they attend: a generate loop's rows are those of the whole sequence turned and prefilled."""
    say("rotary decode loop")
    c, m, n = 16, 2, 80
    p = K.make_params(2, n, c, m, 1, 4, 2, 64)
    lay = K.Layout(p)
    L = lay.aug_len
    r = handle(dict(dim=64, base=1000.0))
    q, k, v = randn(2, L, 4, 64, seed=1), randn(2, L, 2, 64, seed=2), randn(2, L, 2, 64, seed=3)
    want, _ = K.ksa_prefill_fwd(lay, *K.ksa_rotary_fwd(p, r, q, k), v)
    _, rows = K.cache_geometry(p)
    kc, vc = (torch.zeros(2, 2, rows, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for a in range(L):
        j, x = divmod(a, c + m)
        kind, at = (K.KSA_ROW_TEXT, j * c + x) if x < c else (K.KSA_ROW_SUMMARY, j * m + x - c)
        pos = torch.full((2,), at, dtype=torch.int32, device="cuda")
        q1, k1 = K.ksa_rotary_step(p, r, kind, q[:, a], k[:, a], pos)
        K.ksa_cache_append(p, kind, k1.contiguous(), v[:, a].contiguous(), pos, kc, vc)
        o, _ = (K.ksa_decode_fwd if kind == K.KSA_ROW_TEXT else K.ksa_decode_summary_fwd)(p, q1.contiguous(), kc, vc, pos)
        # two kernels' bars against the definition, 2e-2 each
        assert float((o.float() - want[:, a].float()).abs().max()) <= 4e-2, a


def test_python_refuses_single_rows_that_do_not_fit():
    p = K.make_params(2, 100, 16, 2, 1, 4, 2, 128)
    r = handle(RULES[0])
    q, k, pos = randn(2, 4, 128), randn(2, 2, 128), torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in ((q[:1], k, pos), (q, q, pos), (q.float(), k, pos), (None, None, pos), (q, k, pos[:1]), (q, k, pos.long()), (q, k, pos.cpu()), (q.cpu(), k, pos), (None, k, pos, q)):
        with pytest.raises(ValueError):
            K.ksa_rotary_step(p, r, K.KSA_ROW_TEXT, *bad)
    with pytest.raises(K.KsaError):
        K.ksa_rotary_step(p, r, 5, q, k, pos)
