"""Rotary positions without a GPU: frequencies against the formulas, and refusals before any HIP call."""
import ctypes as C
import math
from fractions import Fraction

import pytest

import paper_2604_24432_amd as K
from paper_2604_24432_amd import binding
from tests.rotary import RULES, frequencies, name
from tests.test_paged_host import INVALID, PTR, UNSUPPORTED, cache, params


@pytest.mark.parametrize("rule", RULES, ids=name)
def test_frequencies(rule):
    r = {k: v for k, v in rule.items() if k not in ("interleaved", "magnitude")}
    turns, magnitude = K.rotary_turns(**r)
    want, want_magnitude = frequencies({**r})
    assert len(turns) == rule["dim"] // 2 and magnitude == pytest.approx(want_magnitude, rel=2 ** -24)
    for t, f in zip(turns, want):
        # (a float64 power is off by a few of its 2^-53, and so is 2 pi)
        assert abs(Fraction(int(t), 2 ** 64) - Fraction(f) / Fraction(2 * math.pi)) <= Fraction(f) * Fraction(8, 2 ** 53) + Fraction(1, 2 ** 64)


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=-2), dict(dim=7), dict(dim=8, base=1.0), dict(dim=8, base=math.inf), dict(dim=8, base=math.nan),
                                 dict(dim=8, scaling="linear", factor=0.5), dict(dim=8, scaling="linear", factor=math.nan), dict(dim=8, scaling="by_parts", factor=math.inf),
                                 dict(dim=8, scaling="by_parts", original=0.0), dict(dim=8, scaling="by_parts", slow=-1.0), dict(dim=8, scaling="by_parts", slow=4.0, fast=4.0),
                                 dict(dim=8, scaling="by_parts", fast=math.inf)], ids=name)
def test_rules_that_make_no_sense_are_refused(bad):
    with pytest.raises(K.KsaError) as e:
        K.rotary_turns(**bad)
    assert e.value.status == INVALID


def test_unknown_scalings_and_null_pointers_are_refused():
    with pytest.raises(ValueError):
        K.rotary_turns(8, scaling="other")
    assert binding.lib().ksa_rotary_turns(None, None, None) == INVALID
    rule, out = binding.ksa_rotary_rule(8, 3, 1e4, 1, 1, 1, 32), (C.c_uint64 * 4)()
    assert binding.lib().ksa_rotary_turns(C.byref(rule), out, C.byref(C.c_float())) == INVALID


def rotary(**more):
    f = dict(dim=64, interleaved=0, magnitude=1.0, reserved=0, turns=PTR)
    f.update(more)
    return binding.ksa_rotary(*[f[x] for x, _ in binding.ksa_rotary._fields_])


BAD = [dict(dim=0), dict(dim=130), dict(dim=63), dict(dim=-2), dict(interleaved=2), dict(interleaved=-1), dict(magnitude=0.0), dict(magnitude=-1.0), dict(magnitude=math.inf),
       dict(magnitude=math.nan), dict(reserved=1), dict(turns=None), dict(turns=PTR + 4)]


def whole(entry, p=None, r=None, q=PTR, k=PTR, q_out=PTR, k_out=PTR, qs=None, ks=None, qos=None, kos=None):
    i64 = lambda x: (C.c_int64 * 3)(*x) if x else None  # noqa: E731
    r = rotary() if r is None else r
    return getattr(binding.lib(), entry)(C.byref(params() if p is None else p), C.byref(r) if r else None, q, k, q_out, k_out, i64(qs), i64(ks), i64(qos), i64(kos), None)


@pytest.mark.parametrize("entry", ["ksa_rotary_fwd", "ksa_rotary_bwd"])
def test_whole_sequences_are_refused(entry):
    for bad in BAD:
        assert whole(entry, r=rotary(**bad)) == INVALID, bad
    for bad in (dict(r=False), dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(q=None, k=None, q_out=None, k_out=None), dict(q=PTR + 8), dict(k_out=PTR + 2),
                dict(qs=(0, 128, 128)), dict(ks=(1024, 256, 12)), dict(qos=(1024, -256, 128)), dict(kos=(4, 256, 128))):
        assert whole(entry, **bad) == INVALID, bad
    assert whole(entry, p=params(batch=0)) == INVALID
    assert whole(entry, p=params(head_dim=96)) == UNSUPPORTED
    assert whole(entry, p=params(batch=65535, n_text=1024)) == UNSUPPORTED


def paged(p=None, c=None, r=None, q=PTR, q_out=PTR, k=PTR, v=PTR, qs=None, qos=None, kvs=None, cu=PTR, start=PTR, total=10):
    i64 = lambda x: (C.c_int64 * 2)(*x) if x else None  # noqa: E731
    r = rotary() if r is None else r
    c = cache() if c is None else c
    return binding.lib().ksa_paged_rotary(C.byref(params() if p is None else p), C.byref(c) if c else None, C.byref(r) if r else None, q, q_out, k, v, i64(qs), i64(qos), i64(kvs),
                                          cu, start, total, None)


def test_new_rows_are_refused():
    for bad in BAD:
        assert paged(r=rotary(**bad)) == INVALID, bad
    for bad in (dict(r=False), dict(c=False), dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(q=PTR + 4), dict(q_out=PTR + 8), dict(k=PTR + 8), dict(cu=None), dict(start=None),
                dict(total=-1), dict(qs=(0, 128)), dict(qos=(1024, 12)), dict(kvs=(256, -128)), dict(c=cache(page_rows=12))):
        assert paged(**bad) == INVALID, bad
    assert paged(p=params(head_dim=32)) == UNSUPPORTED
    assert paged(p=params(n_q_heads=1, n_kv_heads=1), total=2 ** 26) == UNSUPPORTED
    assert paged(total=0, q=None, q_out=None, k=None, v=None) == 0


def step(p=None, r=None, kind=0, q=PTR, k=PTR, pos=PTR, q_out=PTR, k_out=PTR, qs=None, ks=None, qos=None, kos=None):
    i64 = lambda x: (C.c_int64 * 2)(*x) if x else None  # noqa: E731
    r = rotary() if r is None else r
    return binding.lib().ksa_rotary_step(C.byref(params() if p is None else p), C.byref(r) if r else None, kind, q, k, pos, q_out, k_out, i64(qs), i64(ks), i64(qos), i64(kos), None)


def test_single_rows_are_refused():
    for bad in BAD:
        assert step(r=rotary(**bad)) == INVALID, bad
    for bad in (dict(r=False), dict(kind=2), dict(kind=-1), dict(kind=1, p=params(n_summary=0)), dict(pos=None), dict(pos=PTR + 2), dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None),
                dict(q=None, k=None, q_out=None, k_out=None), dict(q=PTR + 8), dict(k_out=PTR + 2), dict(qs=(0, 128)), dict(ks=(256, 12)), dict(qos=(1024, -128)), dict(kos=(4, 128))):
        assert step(**bad) == INVALID, bad
    assert step(p=params(batch=0)) == INVALID and step(p=params(head_dim=96)) == UNSUPPORTED


def test_rows_whose_launch_would_have_2_to_the_32_lanes_are_refused():
    """A row takes a wave, four of them a workgroup of 256, and a launch has less than 2^32 lanes: 2^26 - 4 rows are the most."""
    for rows in (2 ** 26 - 3, 2 ** 26 - 2, 2 ** 26 - 1, 2 ** 26):
        p = params(batch=1, n_text=rows, chunk_len=64, n_summary=0)
        for entry in ("ksa_rotary_fwd", "ksa_rotary_bwd"):
            assert whole(entry, p=p) == UNSUPPORTED, (entry, rows)
        assert paged(p=params(n_q_heads=1, n_kv_heads=1), total=rows) == UNSUPPORTED, rows
    for entry in ("ksa_rotary_fwd", "ksa_rotary_bwd"):
        assert whole(entry, p=params(batch=3, n_text=(2 ** 26 - 1) // 3, chunk_len=64, n_summary=0)) == UNSUPPORTED
