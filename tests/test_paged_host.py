"""The paged cache's host side (no GPU needed): refusals before any HIP call, sizes of tables and workspaces, and the kernels' index
functions against the definitions."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2604_24432_amd as K
from paper_2604_24432_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_24432_amd", "csrc")
INVALID, UNSUPPORTED, TOO_SMALL, OUT_OF_RANGE = -1, -2, -3, -5
PTR = 4096          # an aligned address that is never read


def params(**more):
    return K.make_params(**{**dict(batch=2, n_text=1024, chunk_len=64, n_summary=8, window_chunks=1, n_q_heads=8, n_kv_heads=2, head_dim=128), **more})


def cache(fp8=False, **more):
    f = dict(format=1 if fp8 else 0, page_rows=16, n_pages=100, text_pages=64, summary_pages=8, reserved=0, text_table=PTR, summary_table=PTR, k=PTR, v=PTR,
             k_exp=PTR if fp8 else None, v_exp=PTR if fp8 else None, strides=(C.c_int64 * 3)(0, 0, 0))
    f.update(more)
    return binding.ksa_paged_cache(*[f[x] for x, _ in binding.ksa_paged_cache._fields_])


def move(entry, p=None, c=None, k=PTR, v=PTR, strides=None, cu=PTR, start=PTR, total=10):
    p = params() if p is None else p
    c = cache() if c is None else c
    return getattr(binding.lib(), entry)(C.byref(p), C.byref(c) if c else None, k, v, (C.c_int64 * 2)(*strides) if strides else None, cu, start, total, None)


def fwd(p=None, c=None, q=PTR, o=PTR, lse=PTR, qs=None, os_=None, cu=PTR, start=PTR, total=10, most=10, ws=PTR, ws_bytes=0, splits=2):
    p = params() if p is None else p
    c = cache() if c is None else c
    i64 = lambda x: (C.c_int64 * 2)(*x) if x else None  # noqa: E731
    return binding.lib().ksa_paged_fwd(C.byref(p), C.byref(c) if c else None, q, o, lse, i64(qs), i64(os_), cu, start, total, most, ws, ws_bytes, splits, None)


CACHES = [dict(format=2), dict(format=-1), dict(page_rows=0), dict(page_rows=4), dict(page_rows=24), dict(page_rows=2048), dict(n_pages=0), dict(n_pages=-3),
          dict(text_pages=0), dict(text_table=None), dict(summary_pages=0), dict(summary_pages=-1), dict(summary_table=None), dict(text_table=PTR + 2),
          dict(k=None), dict(v=None), dict(k=PTR + 8), dict(v=PTR + 2), dict(k_exp=PTR), dict(v_exp=PTR), dict(reserved=1),
          dict(strides=(C.c_int64 * 3)(0, 128, 128)), dict(strides=(C.c_int64 * 3)(4096, 2048, 4)), dict(strides=(C.c_int64 * 3)(4096, -2048, 128)),
          dict(strides=(C.c_int64 * 3)(2 ** 62 + 2 ** 40, 2048, 128))]


@pytest.mark.parametrize("bad", CACHES, ids=lambda x: "-".join(x))
def test_caches_that_make_no_sense_are_refused(bad):
    c = cache(**bad)
    assert move("ksa_paged_append", c=c) == INVALID and move("ksa_paged_read", c=c) == INVALID and fwd(c=c) == INVALID


def test_an_8_bit_cache_has_exponents_and_strides_of_16_bytes():
    for bad in (dict(k_exp=None), dict(v_exp=None), dict(strides=(C.c_int64 * 3)(8192, 4096, 136))):
        c = cache(fp8=True, **bad)
        assert move("ksa_paged_append", c=c) == INVALID and move("ksa_paged_read", c=c) == INVALID and fwd(c=c) == INVALID


@pytest.mark.parametrize("entry", ["ksa_paged_append", "ksa_paged_read"])
def test_moves_are_refused(entry):
    for bad in (dict(k=None), dict(v=None), dict(k=PTR + 4), dict(cu=None), dict(start=None), dict(cu=PTR + 1), dict(start=PTR + 2), dict(total=-1),
                dict(strides=(0, 128)), dict(strides=(256, 12)), dict(strides=(-256, 128)), dict(c=False)):
        assert move(entry, **bad) == INVALID, bad
    assert move(entry, p=params(head_dim=96)) == UNSUPPORTED
    assert move(entry, p=params(batch=0)) == INVALID
    assert move(entry, total=2 ** 28) == UNSUPPORTED
    assert move(entry, p=params(n_q_heads=1, n_kv_heads=1), total=2 ** 28) == UNSUPPORTED     # more lanes than a launch holds
    assert move(entry, total=0, k=None, v=None) == 0             # nothing to do


def test_attention_is_refused():
    for bad in (dict(q=None), dict(o=None), dict(q=PTR + 8), dict(o=PTR + 2), dict(lse=PTR + 2), dict(cu=None), dict(start=None), dict(total=-1), dict(most=0),
                dict(most=-5), dict(splits=-1), dict(splits=1025), dict(ws=PTR + 8), dict(ws=None), dict(qs=(1024, 4)), dict(os_=(0, 128)), dict(c=False)):
        assert fwd(**bad) == INVALID, bad
    assert fwd() == TOO_SMALL
    assert fwd(p=params(n_q_heads=7)) == INVALID
    assert fwd(p=params(head_dim=32)) == UNSUPPORTED
    assert fwd(total=2 ** 28, splits=1) == UNSUPPORTED
    assert fwd(p=params(n_q_heads=1, n_kv_heads=1), total=2 ** 24, most=2 ** 24, splits=16, ws_bytes=2 ** 62) == UNSUPPORTED
    assert fwd(p=params(batch=60000, n_kv_heads=200, n_q_heads=200), total=10 ** 6, most=10 ** 6, splits=1024, ws_bytes=2 ** 62) == UNSUPPORTED
    assert fwd(total=0, q=None, o=None, ws=None) == 0


def test_workspaces():
    ws = binding.lib().ksa_paged_workspace_bytes
    p = params()
    assert ws(C.byref(p), 10, 10, 1) == 0 and ws(C.byref(p), 0, 10, 4) == 0
    assert ws(C.byref(p), 10, 10, 4) == 10 * 8 * 4 * 132 * 4
    for bad in ((-1, 1, 1), (10, 0, 1), (10, 10, -1), (10, 10, 1025), (2 ** 40, 10, 2)):
        assert ws(C.byref(p), *bad) == 0
    assert ws(C.byref(params(head_dim=7)), 10, 10, 4) == 0
    # what the library chooses by itself stays within a few spans per compute unit
    for batch, total, most, n in ((1, 1, 1, 131072), (64, 64, 1, 131072), (1, 4096, 4096, 131072), (1, 8, 8, 1024), (300, 900, 3, 4096)):
        p = K.make_params(batch, n, 64, 8, 1, 32, 8, 128)
        spans = ws(C.byref(p), total, most, 0) // (total * 32 * 132 * 4)
        assert 0 <= spans <= 1024 and spans != 1


def test_columns_of_the_tables():
    p = params()
    assert K.paged_pages(p, 16, 0) == (0, 0)
    assert K.paged_pages(p, 16, 64) == (4, 0) and K.paged_pages(p, 16, 65) == (4, 1) and K.paged_pages(p, 16, 72 * 3 + 1) == (13, 2)
    assert K.paged_pages(params(n_summary=0), 1024, 1024) == (1, 0)
    for bad, want in (((12, 5), INVALID), ((16, -1), INVALID), ((16, 72 * 16 + 1), OUT_OF_RANGE)):
        with pytest.raises(K.KsaError) as e:
            K.paged_pages(p, *bad)
        assert e.value.status == want


def test_index_functions_against_the_definitions(tmp_path):
    exe = str(tmp_path / "paged_index")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", CSRC,
                    os.path.join(ROOT, "tests", "plan", "paged_index.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr[-2000:]
