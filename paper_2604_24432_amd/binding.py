"""Thin ctypes binding of libksa.so (include/ksa.h).  Argument marshalling only.

Every step of the hot path runs in the library's HIP kernels; this module never computes
attention itself and has no fallback: if libksa.so is missing or a call fails, it raises.
PyTorch is used for device memory and streams only.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass
from typing import Any, NamedTuple, Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("KSA_LIB", os.path.join(_HERE, "libksa.so"))

KSA_FLAG_SUMMARY_SELF_ONLY = 1
KSA_TILE_FULL, KSA_TILE_MASKED = 0, 1
KSA_SPACE_TEXT, KSA_SPACE_SUMMARY = 0, 1


class KsaError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


class ksa_params(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_text", C.c_int32), ("chunk_len", C.c_int32),
                ("n_summary", C.c_int32), ("compress_ratio", C.c_int32), ("window_chunks", C.c_int32),
                ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("softmax_scale", C.c_float), ("flags", C.c_uint32)]


def make_params(batch, n_text, chunk_len, n_summary, window_chunks, n_q_heads, n_kv_heads, head_dim,
                softmax_scale=0.0, flags=0, compress_ratio=None) -> ksa_params:
    if compress_ratio is None:
        compress_ratio = chunk_len // n_summary if n_summary else 0
    return ksa_params(batch, n_text, chunk_len, n_summary, compress_ratio, window_chunks, n_q_heads,
                      n_kv_heads, head_dim, softmax_scale, flags)


class ksa_rotary(C.Structure):
    _fields_ = [("dim", C.c_int32), ("interleaved", C.c_int32), ("magnitude", C.c_float), ("reserved", C.c_int32), ("turns", C.c_void_p)]


class ksa_rotary_rule(C.Structure):
    _fields_ = [("dim", C.c_int32), ("scaling", C.c_int32), ("base", C.c_double), ("factor", C.c_double), ("original", C.c_double), ("slow", C.c_double),
                ("fast", C.c_double)]


_lib = None


def lib():
    """Load libksa.so; raises if it has not been built (python -m paper_2604_24432_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_24432_amd.build` "
                           "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    vp, i32p, i64p, u8p = C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int64), C.POINTER(C.c_uint8)
    pp = C.POINTER(ksa_params)
    sig = {
        "ksa_build_layout": (C.c_int, [pp, C.POINTER(vp)]),
        "ksa_layout_destroy": (None, [vp]),
        "ksa_layout_upload": (C.c_int, [vp]),
        "ksa_augmented_rows": (C.c_int, [pp, C.c_int64, i64p]),
        "ksa_layout_dims": (C.c_int, [vp, i64p, i32p, i32p, i32p, i32p]),
        "ksa_layout_index_maps": (C.c_int, [vp, vp, vp, vp, vp, vp]),
        "ksa_layout_row_ranges": (C.c_int, [vp, C.c_int64, i32p]),
        "ksa_layout_mask_row": (C.c_int, [vp, C.c_int64, vp]),
        "ksa_layout_tile_pairs": (C.c_int, [vp, i64p, vp, vp, vp, vp, vp, vp, vp]),
        "ksa_layout_launch_order": (C.c_int, [vp, i64p, vp, vp, vp, vp]),
        "ksa_prefill_workspace_bytes": (C.c_size_t, [vp]),
        "ksa_prefill_fwd": (C.c_int, [vp, vp, vp, vp, vp, vp, i64p, i64p, i64p, vp, C.c_size_t, vp]),
        "ksa_prefill_relayout_v": (C.c_int, [vp, vp, i64p, vp, C.c_size_t, vp]),
        "ksa_prefill_bwd_workspace_bytes": (C.c_size_t, [vp]),
        "ksa_prefill_bwd": (C.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64p, i64p, i64p, i64p, i64p, vp,
                                      C.c_size_t, vp]),
        "ksa_cache_geometry": (C.c_int, [pp, i32p, i32p]),
        "ksa_cache_text_row": (C.c_int, [pp, C.c_int64, i32p]),
        "ksa_cache_summary_row": (C.c_int, [pp, C.c_int64, i32p]),
        "ksa_decode_ranges": (C.c_int, [pp, C.c_int64, i32p]),
        "ksa_decode_workspace_bytes": (C.c_size_t, [pp, C.c_int32]),
        "ksa_decode_fwd": (C.c_int, [pp, vp, vp, vp, vp, vp, vp, i64p, vp, C.c_size_t, C.c_int32, vp]),
        "ksa_decode_fwd_static": (C.c_int, [pp, vp, vp, vp, vp, vp, vp, i64p, C.c_int32, vp]),
        "ksa_decode_summary_ranges": (C.c_int, [pp, C.c_int64, i32p]),
        "ksa_decode_summary_fwd": (C.c_int, [pp, vp, vp, vp, vp, vp, vp, i64p, vp, C.c_size_t, C.c_int32, vp]),
        "ksa_cache_from_prefill": (C.c_int, [pp, C.c_int64, vp, vp, i64p, vp, vp, i64p, vp]),
        "ksa_cache_append": (C.c_int, [pp, C.c_int32, vp, vp, vp, vp, vp, i64p, vp]),
        "ksa_paged_pages": (C.c_int, [pp, C.c_int32, C.c_int64, i64p, i64p]),
        "ksa_paged_append": (C.c_int, [pp, vp, vp, vp, i64p, vp, vp, C.c_int64, vp]),
        "ksa_paged_read": (C.c_int, [pp, vp, vp, vp, i64p, vp, vp, C.c_int64, vp]),
        "ksa_paged_workspace_bytes": (C.c_size_t, [pp, C.c_int64, C.c_int64, C.c_int32]),
        "ksa_paged_fwd": (C.c_int, [pp, vp, vp, vp, vp, i64p, i64p, vp, vp, C.c_int64, C.c_int64, vp, C.c_size_t, C.c_int32, vp]),
        "ksa_paged_advance_workspace_bytes": (C.c_size_t, [pp, vp]),
        "ksa_paged_advance": (C.c_int, [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, C.c_int64, vp, C.c_size_t, vp]),
        "ksa_rotary_turns": (C.c_int, [C.POINTER(ksa_rotary_rule), C.POINTER(C.c_uint64), C.POINTER(C.c_float)]),
        "ksa_rotary_fwd": (C.c_int, [pp, vp, vp, vp, vp, vp, i64p, i64p, i64p, i64p, vp]),
        "ksa_rotary_bwd": (C.c_int, [pp, vp, vp, vp, vp, vp, i64p, i64p, i64p, i64p, vp]),
        "ksa_rotary_step": (C.c_int, [pp, vp, C.c_int32, vp, vp, vp, vp, vp, i64p, i64p, i64p, i64p, vp]),
        "ksa_paged_rotary": (C.c_int, [pp, vp, vp, vp, vp, vp, vp, i64p, i64p, i64p, vp, vp, C.c_int64, vp]),
        "ksa_status_string": (C.c_char_p, [C.c_int]),
        "ksa_build_info": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)   # AttributeError if the library lacks a declared symbol
        fn.restype, fn.argtypes = res, args
    _lib = L
    return L


EXPORTED_SYMBOLS = ("ksa_augmented_rows", "ksa_build_layout", "ksa_layout_destroy", "ksa_layout_upload", "ksa_layout_dims",
                    "ksa_layout_index_maps", "ksa_layout_row_ranges", "ksa_layout_mask_row",
                    "ksa_layout_tile_pairs", "ksa_layout_launch_order", "ksa_prefill_workspace_bytes", "ksa_prefill_fwd", "ksa_prefill_relayout_v",
                    "ksa_prefill_bwd_workspace_bytes", "ksa_prefill_bwd", "ksa_cache_geometry", "ksa_cache_text_row",
                    "ksa_cache_summary_row", "ksa_decode_ranges", "ksa_decode_workspace_bytes",
                    "ksa_decode_fwd", "ksa_decode_fwd_static", "ksa_decode_summary_ranges", "ksa_decode_summary_fwd", "ksa_cache_from_prefill",
                    "ksa_cache_append", "ksa_paged_pages", "ksa_paged_append", "ksa_paged_read", "ksa_paged_workspace_bytes", "ksa_paged_fwd",
                    "ksa_paged_advance_workspace_bytes", "ksa_paged_advance", "ksa_rotary_turns", "ksa_rotary_fwd", "ksa_rotary_bwd", "ksa_rotary_step", "ksa_paged_rotary", "ksa_status_string", "ksa_build_info")


def status_string(status: int) -> str:
    return lib().ksa_status_string(status).decode()


def build_info() -> str:
    return lib().ksa_build_info().decode()


def _check(rc: int, what: str):
    if rc != 0:
        raise KsaError(rc, what)


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


class Layout:
    """Owner of a ksa_layout* (freed on garbage collection)."""

    def __init__(self, params: ksa_params):
        self.params = params
        h = C.c_void_p()
        _check(lib().ksa_build_layout(C.byref(params), C.byref(h)), "ksa_build_layout")
        self._h = h
        L, J, qt, kt, hs = C.c_int64(), C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32()
        _check(lib().ksa_layout_dims(h, C.byref(L), C.byref(J), C.byref(qt), C.byref(kt), C.byref(hs)),
               "ksa_layout_dims")
        self.aug_len, self.n_chunks, self.q_tile_rows, self.k_tile_rows = L.value, J.value, qt.value, kt.value
        self.heads_per_workgroup = hs.value

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h:
            lib().ksa_layout_destroy(h)

    @property
    def handle(self):
        return self._h

    def upload(self):
        _check(lib().ksa_layout_upload(self._h), "ksa_layout_upload")

    def index_maps(self):
        p = self.params
        out = dict(aug_chunk=np.zeros(self.aug_len, np.int32), aug_is_summary=np.zeros(self.aug_len, np.uint8),
                   position_ids=np.zeros(self.aug_len, np.int32), text_to_aug=np.zeros(p.n_text, np.int32),
                   summary_to_aug=np.zeros(self.n_chunks * p.n_summary, np.int32))
        _check(lib().ksa_layout_index_maps(self._h, *[_np_ptr(out[k]) for k in
               ("aug_chunk", "aug_is_summary", "position_ids", "text_to_aug", "summary_to_aug")]), "ksa_layout_index_maps")
        return out

    def row_ranges(self, aq: int) -> np.ndarray:
        out = (C.c_int32 * 4)()
        _check(lib().ksa_layout_row_ranges(self._h, aq, out), "ksa_layout_row_ranges")
        return np.array(out[:], np.int32)

    def mask_row(self, aq: int) -> np.ndarray:
        out = np.zeros(self.aug_len, np.uint8)
        _check(lib().ksa_layout_mask_row(self._h, aq, _np_ptr(out)), "ksa_layout_mask_row")
        return out

    def tile_pairs(self):
        n = C.c_int64()
        _check(lib().ksa_layout_tile_pairs(self._h, C.byref(n), None, None, None, None, None, None, None),
               "ksa_layout_tile_pairs")
        N = n.value
        out = dict(q_space=np.zeros(N, np.uint8), q_begin=np.zeros(N, np.int32), q_count=np.zeros(N, np.int32),
                   k_space=np.zeros(N, np.uint8), k_begin=np.zeros(N, np.int32), k_count=np.zeros(N, np.int32),
                   kind=np.zeros(N, np.uint8))
        _check(lib().ksa_layout_tile_pairs(self._h, C.byref(n), *[_np_ptr(out[k]) for k in
               ("q_space", "q_begin", "q_count", "k_space", "k_begin", "k_count", "kind")]), "ksa_layout_tile_pairs")
        return out


    def launch_order(self):
        n = C.c_int64()
        _check(lib().ksa_layout_launch_order(self._h, C.byref(n), None, None, None, None), "ksa_layout_launch_order")
        N = n.value
        out = dict(q_space=np.zeros(N, np.uint8), q_begin=np.zeros(N, np.int32), batch=np.zeros(N, np.int32),
                   q_head=np.zeros(N, np.int32))
        _check(lib().ksa_layout_launch_order(self._h, C.byref(n), *[_np_ptr(out[k]) for k in
               ("q_space", "q_begin", "batch", "q_head")]), "ksa_layout_launch_order")
        return out


def ksa_build_layout(params: ksa_params) -> Layout:
    return Layout(params)


# ---- torch-facing wrappers ------------------------------------------------------------------------

# The smallest problems (512 tokens, a summary step) take as long as the host needs to hand them over: addresses go to the
# library as plain ints, and the raw stream comes from torch's C interface (0.2 us; a torch.cuda.Stream object 3.3 us).

_I64x3 = C.c_int64 * 3


def _stream_ptr(stream):
    if stream is not None:
        return stream.cuda_stream
    from torch import _C
    return _C._cuda_getCurrentRawStream(_C._cuda_getDevice())


def _strides3(t):
    return _I64x3(*t.stride()[:3])


def _require(t, name, dtype, ndim):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype is not dtype or t.ndim != ndim or t.stride(-1) != 1:
        raise ValueError(f"{name}: expected {ndim}-d {dtype} with contiguous last dim, got {t.dtype} {tuple(t.shape)}")


# A decode step takes less time on the GPU than the checks of its arguments one by one (summary step, batch 16: 8.1 us on the GPU, 17.4
# per step; 5 of the 8.6 us of each call went into checks).  The calls of the decode loop therefore ask first whether everything is
# as it should be, in as few steps as possible (14.6 per step); if not, the checks below say what is wrong.
_FIELDS = struct.Struct("=9i")   # the integers at the front of ksa_params


def _plain_tensors(tensors, dtype) -> bool:
    import torch
    for t in tensors:
        if type(t) is not torch.Tensor or t.dtype is not dtype or not t.is_cuda:
            return False
    return True


def _cache_as_it_should_be(fields, k_cache, v_cache):
    """The caches' strides for the library, or None if something about them is not what the parameters say."""
    batch, n_text, c, m, _, window, _, n_kv_heads, d = fields
    strides = k_cache.stride()
    if c <= 0 or strides != v_cache.stride() or k_cache.shape != v_cache.shape or \
            k_cache.shape != (batch, n_kv_heads, n_text // c * m + (window + 1) * c, d):
        return None
    s0, s1, s2, s3 = strides
    return _I64x3(s0, s1, s2) if s3 == 1 else None


def _same_strides(x, y) -> bool:
    """Strides agree wherever they matter (a dimension of size 1 may carry any stride)."""
    return x.stride() == y.stride() or all(sx == sy for n, sx, sy in zip(x.shape, x.stride(), y.stride()) if n > 1)


def prefill_workspace_bytes(layout: Layout) -> int:
    return int(lib().ksa_prefill_workspace_bytes(layout.handle))


def ksa_prefill_fwd(layout: Layout, q, k, v, o=None, lse=None, return_lse=True, workspace=None, stream=None):
    """q [B, L, Hq, d], k/v [B, L, Hkv, d] bf16 on the GPU -> o [B, L, Hq, d] bf16, lse [B, Hq, L] fp32.
    workspace: uint8 GPU tensor of at least prefill_workspace_bytes(layout) bytes (allocated here if omitted)."""
    import torch
    p = layout.params
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, name, torch.bfloat16, 4)
    if tuple(q.shape) != (p.batch, layout.aug_len, p.n_q_heads, p.head_dim):
        raise ValueError(f"q shape {tuple(q.shape)} does not match the layout")
    if tuple(k.shape) != (p.batch, layout.aug_len, p.n_kv_heads, p.head_dim) or k.shape != v.shape or not _same_strides(k, v):
        raise ValueError("k / v shape or strides do not match the layout")
    if o is None:
        o = torch.empty_like(q)
    _require(o, "o", torch.bfloat16, 4)
    if lse is None and return_lse:
        lse = torch.empty((p.batch, p.n_q_heads, layout.aug_len), dtype=torch.float32, device=q.device)
    lse_ptr = lse.data_ptr() if lse is not None else None
    if workspace is None:
        workspace = torch.empty(prefill_workspace_bytes(layout), dtype=torch.uint8, device=q.device)
    if not workspace.is_cuda or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 GPU tensor")
    rc = lib().ksa_prefill_fwd(layout.handle, q.data_ptr(), k.data_ptr(),
                               v.data_ptr(), o.data_ptr(), lse_ptr,
                               _strides3(q), _strides3(k), _strides3(o),
                               workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    _check(rc, "ksa_prefill_fwd")
    return o, lse


def ksa_prefill_relayout_v(layout: Layout, v, workspace, stream=None):
    """Only the first kernel of ksa_prefill_fwd (key-major copy of V into the workspace); for timing."""
    import torch
    _require(v, "v", torch.bfloat16, 4)
    rc = lib().ksa_prefill_relayout_v(layout.handle, v.data_ptr(), _strides3(v),
                                      workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    _check(rc, "ksa_prefill_relayout_v")


def prefill_bwd_workspace_bytes(layout: Layout) -> int:
    return int(lib().ksa_prefill_bwd_workspace_bytes(layout.handle))


def ksa_prefill_bwd(layout: Layout, q, k, v, o, lse, d_o, dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Gradients of ksa_prefill_fwd: q, o, d_o [B, L, Hq, d], k/v [B, L, Hkv, d] bf16, lse [B, Hq, L] fp32 on the GPU
    -> dq like q, dk and dv like k.  o and d_o must share their strides."""
    import torch
    p = layout.params
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (o, "o"), (d_o, "d_o")):
        _require(t, name, torch.bfloat16, 4)
    _require(lse, "lse", torch.float32, 3)
    if tuple(q.shape) != (p.batch, layout.aug_len, p.n_q_heads, p.head_dim) or o.shape != q.shape or d_o.shape != q.shape:
        raise ValueError(f"q / o / d_o shape {tuple(q.shape)} does not match the layout")
    if tuple(k.shape) != (p.batch, layout.aug_len, p.n_kv_heads, p.head_dim) or k.shape != v.shape or not _same_strides(k, v):
        raise ValueError("k / v shape or strides do not match the layout")
    if not _same_strides(o, d_o):
        raise ValueError("o and d_o must have the same strides")
    if tuple(lse.shape) != (p.batch, p.n_q_heads, layout.aug_len) or not lse.is_contiguous():
        raise ValueError("lse must be contiguous [B, Hq, L]")
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(dk) if dv is None else dv
    for t, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        _require(t, name, torch.bfloat16, 4)
    if dq.shape != q.shape or dk.shape != k.shape or dv.shape != k.shape or not _same_strides(dk, dv):
        raise ValueError("dq / dk / dv shape or strides do not match q / k / v")
    if workspace is None:
        workspace = torch.empty(prefill_bwd_workspace_bytes(layout), dtype=torch.uint8, device=q.device)
    if not workspace.is_cuda or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 GPU tensor")
    rc = lib().ksa_prefill_bwd(layout.handle, q.data_ptr(), k.data_ptr(),
                               v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                               d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                               dv.data_ptr(), _strides3(q), _strides3(k),
                               _strides3(o), _strides3(dq), _strides3(dk),
                               workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    _check(rc, "ksa_prefill_bwd")
    return dq, dk, dv


def augmented_rows(params: ksa_params, n_text: int) -> int:
    """Rows of the augmented sequence of n_text text tokens (from the library)."""
    rows = C.c_int64()
    _check(lib().ksa_augmented_rows(C.byref(params), n_text, C.byref(rows)), "ksa_augmented_rows")
    return rows.value


def cache_geometry(params: ksa_params) -> Tuple[int, int]:
    s, r = C.c_int32(), C.c_int32()
    rc = lib().ksa_cache_geometry(params, s, r)
    if rc:
        _check(rc, "ksa_cache_geometry")
    return s.value, r.value


def cache_text_row(params: ksa_params, i: int) -> int:
    r = C.c_int32()
    _check(lib().ksa_cache_text_row(C.byref(params), i, C.byref(r)), "ksa_cache_text_row")
    return r.value


def cache_summary_row(params: ksa_params, u: int) -> int:
    r = C.c_int32()
    _check(lib().ksa_cache_summary_row(C.byref(params), u, C.byref(r)), "ksa_cache_summary_row")
    return r.value


def ksa_decode_ranges(params: ksa_params, pos: int) -> np.ndarray:
    out = (C.c_int32 * 6)()
    _check(lib().ksa_decode_ranges(C.byref(params), pos, out), "ksa_decode_ranges")
    return np.array(out[:], np.int32)


def decode_workspace_bytes(params: ksa_params, n_splits: int = 0) -> int:
    return int(lib().ksa_decode_workspace_bytes(C.byref(params), n_splits))


def _decode_checks(params: ksa_params, q, k_cache, v_cache, pos):
    import torch
    _require(q, "q", torch.bfloat16, 3)
    _require(k_cache, "k_cache", torch.bfloat16, 4)
    _require(v_cache, "v_cache", torch.bfloat16, 4)
    _require(pos, "pos", torch.int32, 1)
    if not q.is_contiguous():
        raise ValueError("q must be contiguous")
    s_cap, rows = cache_geometry(params)
    if tuple(k_cache.shape) != (params.batch, params.n_kv_heads, rows, params.head_dim) or \
            k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride():
        raise ValueError(f"cache shape must be {(params.batch, params.n_kv_heads, rows, params.head_dim)}")
    if tuple(q.shape) != (params.batch, params.n_q_heads, params.head_dim) or pos.shape[0] != params.batch:
        raise ValueError("q / pos shape does not match params")
    return _strides3(k_cache)


def _decode(entry, params: ksa_params, q, k_cache, v_cache, pos, o, lse, return_lse, workspace, n_splits, stream):
    import torch
    cache_strides = None
    if _plain_tensors((q, k_cache, v_cache), torch.bfloat16) and _plain_tensors((pos,), torch.int32):
        fields = _FIELDS.unpack_from(params)
        if q.shape == (fields[0], fields[6], fields[8]) and pos.shape == (fields[0],) and q.is_contiguous() and pos.stride() == (1,):
            cache_strides = _cache_as_it_should_be(fields, k_cache, v_cache)
    if cache_strides is None:
        cache_strides = _decode_checks(params, q, k_cache, v_cache, pos)
    if o is None:
        o = torch.empty_like(q)
    if lse is None and return_lse:
        lse = torch.empty((params.batch, params.n_q_heads), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.empty(decode_workspace_bytes(params, n_splits), dtype=torch.uint8, device=q.device)
    rc = getattr(lib(), entry)(C.byref(params), q.data_ptr(), k_cache.data_ptr(),
                               v_cache.data_ptr(), pos.data_ptr(), o.data_ptr(),
                               lse.data_ptr() if lse is not None else None,
                               cache_strides, workspace.data_ptr(),
                               workspace.numel() * workspace.element_size(), n_splits, _stream_ptr(stream))
    if rc:
        cache_geometry(params)   # (parameters that make no sense are reported under this name)
        _check(rc, entry)
    return o, lse


def ksa_decode_fwd(params: ksa_params, q, k_cache, v_cache, pos, o=None, lse=None, return_lse=True,
                   workspace=None, n_splits: int = 0, stream=None):
    """q [B, Hq, d] bf16; caches [B, Hkv, cache_rows, d] bf16; pos int32 [B] on the GPU (text indices)."""
    return _decode("ksa_decode_fwd", params, q, k_cache, v_cache, pos, o, lse, return_lse, workspace, n_splits, stream)


KSA_DECODE_STATIC_SCRATCH_BYTES = 8 << 20


def ksa_decode_fwd_static(params: ksa_params, q, k_cache, v_cache, pos, o, lse=None, n_splits: int = 0, stream=None):
    """ksa_decode_fwd with the spans' partial records in the library's static device array: the call allocates
    nothing, so o (and lse, if wanted) must be passed in.  Raises KsaError (scratch limit) for problems whose
    records exceed KSA_DECODE_STATIC_SCRATCH_BYTES."""
    import torch
    _require(q, "q", torch.bfloat16, 3)
    _require(o, "o", torch.bfloat16, 3)
    _require(pos, "pos", torch.int32, 1)
    _check_cache(params, k_cache, v_cache)
    if not q.is_contiguous() or not o.is_contiguous() or o.shape != q.shape:
        raise ValueError("q and o must be contiguous and of one shape")
    if tuple(q.shape) != (params.batch, params.n_q_heads, params.head_dim) or pos.shape[0] != params.batch:
        raise ValueError("q / pos shape does not match params")
    if lse is not None:
        _require(lse, "lse", torch.float32, 2)
        if tuple(lse.shape) != (params.batch, params.n_q_heads) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous [B, Hq] tensor")
    rc = lib().ksa_decode_fwd_static(C.byref(params), q.data_ptr(), k_cache.data_ptr(),
                                     v_cache.data_ptr(), pos.data_ptr(),
                                     o.data_ptr(), lse.data_ptr() if lse is not None else None,
                                     _strides3(k_cache), n_splits, _stream_ptr(stream))
    _check(rc, "ksa_decode_fwd_static")
    return o, lse


def ksa_decode_summary_fwd(params: ksa_params, q, k_cache, v_cache, ordinal, o=None, lse=None, return_lse=True,
                           workspace=None, n_splits: int = 0, stream=None):
    """The summary-token step: as ksa_decode_fwd with ordinal int32 [B] = summary ordinals j*m + slot."""
    return _decode("ksa_decode_summary_fwd", params, q, k_cache, v_cache, ordinal, o, lse, return_lse, workspace,
                   n_splits, stream)


def ksa_decode_summary_ranges(params: ksa_params, ordinal: int) -> np.ndarray:
    out = (C.c_int32 * 4)()
    _check(lib().ksa_decode_summary_ranges(C.byref(params), ordinal, out), "ksa_decode_summary_ranges")
    return np.array(out[:], np.int32)


KSA_ROW_TEXT, KSA_ROW_SUMMARY = 0, 1


def _check_cache(params, k_cache, v_cache):
    import torch
    _require(k_cache, "k_cache", torch.bfloat16, 4)
    _require(v_cache, "v_cache", torch.bfloat16, 4)
    s_cap, rows = cache_geometry(params)
    if tuple(k_cache.shape) != (params.batch, params.n_kv_heads, rows, params.head_dim) or \
            k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride():
        raise ValueError(f"cache shape must be {(params.batch, params.n_kv_heads, rows, params.head_dim)}")


def ksa_cache_from_prefill(params: ksa_params, n_prefill: int, k, v, k_cache, v_cache, stream=None):
    """k, v [B, L, Hkv, d] bf16: augmented sequence of n_prefill text tokens; fills the caches in place."""
    import torch
    _require(k, "k", torch.bfloat16, 4)
    _require(v, "v", torch.bfloat16, 4)
    _check_cache(params, k_cache, v_cache)
    L = augmented_rows(params, n_prefill)
    if tuple(k.shape) != (params.batch, L, params.n_kv_heads, params.head_dim) or k.shape != v.shape or \
            k.stride() != v.stride() or k.stride(3) != 1:
        raise ValueError(f"k / v shape must be {(params.batch, L, params.n_kv_heads, params.head_dim)}")
    rc = lib().ksa_cache_from_prefill(C.byref(params), n_prefill, k.data_ptr(), v.data_ptr(),
                                      _strides3(k), k_cache.data_ptr(),
                                      v_cache.data_ptr(), _strides3(k_cache), _stream_ptr(stream))
    _check(rc, "ksa_cache_from_prefill")


def ksa_cache_append(params: ksa_params, kind: int, k_new, v_new, pos, k_cache, v_cache, stream=None):
    """k_new, v_new [B, Hkv, d] bf16 contiguous; pos int32 [B] on the GPU (text indices or summary ordinals)."""
    import torch
    cache_strides = None
    if _plain_tensors((k_new, v_new, k_cache, v_cache), torch.bfloat16) and _plain_tensors((pos,), torch.int32):
        fields = _FIELDS.unpack_from(params)
        rows = (fields[0], fields[7], fields[8])
        if k_new.shape == rows and v_new.shape == rows and pos.shape == rows[:1] and k_new.is_contiguous() and v_new.is_contiguous() and \
                pos.stride() == (1,):
            cache_strides = _cache_as_it_should_be(fields, k_cache, v_cache)
    if cache_strides is None:
        cache_strides = _append_checks(params, k_new, v_new, pos, k_cache, v_cache)
    rc = lib().ksa_cache_append(C.byref(params), kind, k_new.data_ptr(), v_new.data_ptr(),
                                pos.data_ptr(), k_cache.data_ptr(),
                                v_cache.data_ptr(), cache_strides, _stream_ptr(stream))
    if rc:
        cache_geometry(params)
        _check(rc, "ksa_cache_append")


def _append_checks(params: ksa_params, k_new, v_new, pos, k_cache, v_cache):
    import torch
    _require(k_new, "k_new", torch.bfloat16, 3)
    _require(v_new, "v_new", torch.bfloat16, 3)
    _require(pos, "pos", torch.int32, 1)
    _check_cache(params, k_cache, v_cache)
    if tuple(k_new.shape) != (params.batch, params.n_kv_heads, params.head_dim) or k_new.shape != v_new.shape or \
            not k_new.is_contiguous() or not v_new.is_contiguous() or pos.shape[0] != params.batch:
        raise ValueError("k_new / v_new / pos shape does not match params")
    return _strides3(k_cache)


KSA_CACHE_BF16, KSA_CACHE_FP8, KSA_CACHE_FP4 = 0, 1, 2


class ksa_paged_cache(C.Structure):
    _fields_ = [("format", C.c_int32), ("page_rows", C.c_int32), ("n_pages", C.c_int32), ("text_pages", C.c_int32),
                ("summary_pages", C.c_int32), ("reserved", C.c_int32), ("text_table", C.c_void_p), ("summary_table", C.c_void_p),
                ("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p), ("strides", C.c_int64 * 3)]


class PagedCache:
    """A batch of sequences whose K / V rows lie in the pages of one pool (struct ksa_paged_cache); holds its tensors.

    k, v: [n_pages, Hkv, page_rows, d] on the GPU, bfloat16, or float8_e4m3fn with k_exp, v_exp uint8 [n_pages, Hkv, page_rows], or 4-bit floats, two to a
    byte: uint8 [n_pages, Hkv, page_rows, d / 2] with k_exp, v_exp uint8 [n_pages, Hkv, page_rows, d / 32], each at a multiple of 4 bytes.
    text_table, summary_table: int32 [batch, columns], contiguous; their contents may change from call to call.  Other tensors, or other
    parameters, take another PagedCache.  A cache carries no gradient: what is appended, read or attended to is not recorded for autograd.
    """

    def __init__(self, params: ksa_params, k, v, text_table, summary_table=None, k_exp=None, v_exp=None):
        import torch
        params = ksa_params.from_buffer_copy(params)
        f8, f4 = k.dtype is torch.float8_e4m3fn, k.dtype is torch.uint8
        for t, name in ((k, "k"), (v, "v")):
            _require(t, name, torch.float8_e4m3fn if f8 else torch.uint8 if f4 else torch.bfloat16, 4)
        n_pages, heads, rows, d = k.shape
        if (heads, d) != (params.n_kv_heads, params.head_dim // 2 if f4 else params.head_dim) or k.shape != v.shape or not _same_strides(k, v):
            raise ValueError(f"k / v shape must be [n_pages, {params.n_kv_heads}, page_rows, {params.head_dim}{' / 2' if f4 else ''}], with the same strides")
        if (f8 or f4) != (k_exp is not None) or (f8 or f4) != (v_exp is not None):
            raise ValueError("k_exp and v_exp belong to a float8_e4m3fn or 4-bit (uint8) cache, and to no other")
        exps = (n_pages, heads, rows, params.head_dim // 32) if f4 else (n_pages, heads, rows)
        for t, name in ((k_exp, "k_exp"), (v_exp, "v_exp")) if f8 or f4 else ():
            _require(t, name, torch.uint8, len(exps))
            if tuple(t.shape) != exps or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous {exps}")
        if params.n_summary > 0 and summary_table is None:
            raise ValueError("summary_table is missing")
        for t, name in ((text_table, "text_table"), (summary_table, "summary_table")):
            if t is not None:
                _require(t, name, torch.int32, 2)
                if t.shape[0] != params.batch or not t.is_contiguous():
                    raise ValueError(f"{name} must be contiguous with {params.batch} rows")
        tensors = [t for t in (k, v, text_table, summary_table, k_exp, v_exp) if t is not None]
        if any(t.device != k.device for t in tensors):
            raise ValueError("the cache's tensors lie on different devices")
        self.params, self.device = params, k.device
        self.k, self.v, self.text_table, self.summary_table, self.k_exp, self.v_exp = k, v, text_table, summary_table, k_exp, v_exp
        ptr = [t.data_ptr() if t is not None else None for t in (text_table, summary_table, k, v, k_exp, v_exp)]
        self.struct = ksa_paged_cache(KSA_CACHE_FP8 if f8 else KSA_CACHE_FP4 if f4 else KSA_CACHE_BF16, rows, n_pages, text_table.shape[1],
                                      summary_table.shape[1] if summary_table is not None else 0, 0, *ptr, _strides_of(k))

        # what a call needs of all this, as it needs it
        self._args = (C.byref(params), C.byref(self.struct))
        self._dev, self._batch = k.device.index, ((params.batch + 1,), (params.batch,))
        self._kv, self._q = (params.n_kv_heads, params.head_dim), (params.n_q_heads, params.head_dim)

    @property
    def page_rows(self) -> int:
        return self.struct.page_rows

    def _plain(self, x, y, row, cu_rows, start) -> bool:
        """Whether x and y are contiguous [rows, *row] tensors and the batch is as it should be, on the cache's device: in as few steps as possible."""
        import torch
        dev, shape = self._dev, x.shape
        return (x.dtype is torch.bfloat16 and y.dtype is torch.bfloat16 and cu_rows.dtype is torch.int32 and start.dtype is torch.int32 and
                shape == y.shape and shape[1:] == row and (cu_rows.shape, start.shape) == self._batch and x.is_contiguous() and y.is_contiguous() and
                cu_rows.is_contiguous() and start.is_contiguous() and
                x.get_device() == dev and y.get_device() == dev and cu_rows.get_device() == dev and start.get_device() == dev)


def _strides_of(t):
    """Strides for the library: those of dimensions of size 1, which may be anything, as in a contiguous tensor."""
    strides, size = [], t.stride(-1) * t.shape[-1]
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        strides.insert(0, size if n == 1 else s)
        size = strides[0] * n
    return (C.c_int64 * len(strides))(*strides)


def paged_pages(params: ksa_params, page_rows: int, n_rows: int) -> Tuple[int, int]:
    """Columns that text_table and summary_table need for the first n_rows augmented rows of a sequence."""
    t, s = C.c_int64(), C.c_int64()
    _check(lib().ksa_paged_pages(C.byref(params), page_rows, n_rows, C.byref(t), C.byref(s)), "ksa_paged_pages")
    return t.value, s.value


def paged_workspace_bytes(cache: PagedCache, total_rows: int, max_rows: int, n_splits: int = 0) -> int:
    return int(lib().ksa_paged_workspace_bytes(C.byref(cache.params), total_rows, max_rows, n_splits))


def _rows_of_call(cache: PagedCache, tensors, heads, cu_rows, start):
    """Checks the tensors [rows, heads, d] and the batch of a call."""
    import torch
    d = cache.params.head_dim
    for t, name in tensors:
        _require(t, name, torch.bfloat16, 3)
        if tuple(t.shape) != (tensors[0][0].shape[0], heads, d):
            raise ValueError(f"{name}: expected [rows, {heads}, {d}], got {tuple(t.shape)}")
    for t, name, n in ((cu_rows, "cu_rows", cache.params.batch + 1), (start, "start", cache.params.batch)):
        _require(t, name, torch.int32, 1)
        if t.shape[0] != n:
            raise ValueError(f"{name} must have {n} elements")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    if any(t.device != cache.device for t, _ in tensors) or cu_rows.device != cache.device or start.device != cache.device:
        raise ValueError("tensors lie on another device than the cache")


def _check_stream(cache: PagedCache, stream):
    if stream.device != cache.device:
        raise ValueError("stream belongs to another device than the cache")


def _on_device(dev, name, stream, *args):
    """The call on device `dev`: on `stream`, or on that device's current one."""
    from torch import _C
    here = _C._cuda_getDevice()
    if stream is None:
        raw = _C._cuda_getCurrentRawStream(dev)
    elif stream.device.index != dev:
        raise ValueError("stream belongs to another device than the tensors")
    else:
        raw = stream.cuda_stream
    if here == dev:
        rc = getattr(lib(), name)(*args, raw)
    else:
        _C._cuda_setDevice(dev)
        try:
            rc = getattr(lib(), name)(*args, raw)
        finally:
            _C._cuda_setDevice(here)
    if rc:
        _check(rc, name)


def _paged(cache: PagedCache, name, stream, *args):
    """The call, on the cache's device."""
    if stream is not None:
        _check_stream(cache, stream)
    _on_device(cache._dev, name, stream, *cache._args, *args)


def ksa_paged_append(cache: PagedCache, k_new, v_new, cu_rows, start, stream=None):
    """k_new, v_new [rows, Hkv, d] bf16: rows [cu_rows[b], cu_rows[b + 1]) become sequence b's augmented rows from start[b] on.
    cu_rows int32 [batch + 1] and start int32 [batch] lie on the GPU."""
    strides = None
    if not cache._plain(k_new, v_new, cache._kv, cu_rows, start):
        _rows_of_call(cache, ((k_new, "k_new"), (v_new, "v_new")), cache.params.n_kv_heads, cu_rows, start)
        if not _same_strides(k_new, v_new):
            raise ValueError("k_new and v_new must have the same strides")
        strides = _strides_of(k_new)
    _paged(cache, "ksa_paged_append", stream, k_new.data_ptr(), v_new.data_ptr(), strides, cu_rows.data_ptr(), start.data_ptr(), k_new.shape[0])


def ksa_paged_read(cache: PagedCache, cu_rows, start, total_rows: int, k=None, v=None, stream=None):
    """The rows that ksa_paged_append with these cu_rows and start would write -> k, v [total_rows, Hkv, d] bf16.
    What is allocated here belongs to `stream`."""
    import torch
    if stream is not None and (k is None or v is None):
        _check_stream(cache, stream)
        with torch.cuda.stream(stream):
            return ksa_paged_read(cache, cu_rows, start, total_rows, k, v)
    if k is None:
        k = torch.empty((total_rows, *cache._kv), dtype=torch.bfloat16, device=cache.device)
    if v is None:
        v = torch.empty_like(k)
    strides = None
    if not cache._plain(k, v, cache._kv, cu_rows, start):
        _rows_of_call(cache, ((k, "k"), (v, "v")), cache.params.n_kv_heads, cu_rows, start)
        if not _same_strides(k, v):
            raise ValueError("k and v must have the same strides")
        strides = _strides_of(k)
    if k.shape[0] != total_rows:
        raise ValueError(f"k and v must have {total_rows} rows")
    _paged(cache, "ksa_paged_read", stream, k.data_ptr(), v.data_ptr(), strides, cu_rows.data_ptr(), start.data_ptr(), total_rows)
    return k, v


def ksa_paged_fwd(cache: PagedCache, q, cu_rows, start, max_rows: Optional[int] = None, o=None, lse=None, return_lse=True, workspace=None,
                  n_splits: int = 0, stream=None):
    """q [rows, Hq, d] bf16, the queries of the rows that ksa_paged_append wrote -> o like q, lse [rows, Hq] fp32; no gradients.
    max_rows: the largest number of rows of a sequence; omitted it is all of them, with which single rows of several sequences take the kernel for
    many rows (64 sequences 1.2 to 2.3 times as long); workspace: uint8, at least
    paged_workspace_bytes(cache, rows, max_rows, n_splits) bytes (allocated here if omitted; with n_splits = 0 a smaller one, of any size, means
    fewer spans).  What is allocated here belongs to `stream`."""
    import torch
    if stream is not None and (o is None or workspace is None or lse is None and return_lse):
        _check_stream(cache, stream)
        with torch.cuda.stream(stream):
            return ksa_paged_fwd(cache, q, cu_rows, start, max_rows, o, lse, return_lse, workspace, n_splits)
    rows = q.shape[0]
    if max_rows is None:
        max_rows = max(rows, 1)
    if o is None:
        o = torch.empty_like(q)
    q_strides = o_strides = None
    if not cache._plain(q, o, cache._q, cu_rows, start):
        _rows_of_call(cache, ((q, "q"), (o, "o")), cache.params.n_q_heads, cu_rows, start)
        q_strides, o_strides = _strides_of(q), _strides_of(o)
    if lse is None:
        if return_lse:
            lse = q.new_empty((rows, cache.params.n_q_heads), dtype=torch.float32)
    else:
        _require(lse, "lse", torch.float32, 2)
        if tuple(lse.shape) != (rows, cache.params.n_q_heads) or not lse.is_contiguous() or lse.device != cache.device:
            raise ValueError(f"lse must be contiguous {(rows, cache.params.n_q_heads)} on the cache's device")
    if workspace is None:
        workspace = torch.empty(paged_workspace_bytes(cache, rows, max_rows, n_splits), dtype=torch.uint8, device=cache.device)
    elif workspace.dtype is not torch.uint8 or workspace.get_device() != cache._dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the cache's device")
    _paged(cache, "ksa_paged_fwd", stream, q.data_ptr(), o.data_ptr(), lse.data_ptr() if lse is not None else None, q_strides, o_strides,
           cu_rows.data_ptr(), start.data_ptr(), rows, max_rows, workspace.data_ptr(), workspace.numel(), n_splits)
    return o, lse


# ---- rotary positions --------------------------------------------------------------------------------

KSA_ROTARY_PLAIN, KSA_ROTARY_LINEAR, KSA_ROTARY_BY_PARTS = 0, 1, 2
_SCALINGS = {None: KSA_ROTARY_PLAIN, "linear": KSA_ROTARY_LINEAR, "by_parts": KSA_ROTARY_BY_PARTS}


def rotary_turns(dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0, original: float = 1.0, slow: float = 1.0,
                 fast: float = 32.0) -> Tuple[np.ndarray, float]:
    """The frequencies of a rule, uint64 [dim / 2] in turns per position times 2^64, and its magnitude (struct ksa_rotary_rule)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {tuple(_SCALINGS)}")
    turns, magnitude = np.zeros(max(dim // 2, 1), np.uint64), C.c_float()
    rule = ksa_rotary_rule(dim, _SCALINGS[scaling], base, factor, original, slow, fast)
    _check(lib().ksa_rotary_turns(C.byref(rule), turns.ctypes.data_as(C.POINTER(C.c_uint64)), C.byref(magnitude)), "ksa_rotary_turns")
    return turns, magnitude.value


class Rotary:
    """Rotary positions (struct ksa_rotary): the first `dim` elements of a head are turned in pairs, (2i, 2i + 1) if interleaved, else (i, i + dim / 2), by
    position * base^(-2i / dim).  scaling: None; "linear" (all frequencies divided by factor); "by_parts" (those that turn less than `slow` times
    over `original` positions are, those that turn more than `fast` times are not, between them in proportion).  magnitude scales what is turned; None: 1, by
    parts 0.1 ln(factor) + 1.  Holds the frequencies on the device."""

    def __init__(self, dim: int, base: float = 10000.0, interleaved: bool = False, scaling: Optional[str] = None, factor: float = 1.0, original: float = 1.0,
                 slow: float = 1.0, fast: float = 32.0, magnitude: Optional[float] = None, device="cuda"):
        import torch
        turns, by_rule = rotary_turns(dim, base, scaling, factor, original, slow, fast)
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        if not self.turns.is_cuda:
            raise ValueError("device must be a GPU")
        self.device, self._dev = self.turns.device, self.turns.device.index
        self.struct = ksa_rotary(dim, 1 if interleaved else 0, by_rule if magnitude is None else magnitude, 0, self.turns.data_ptr())
        self._arg = C.byref(self.struct)

    @property
    def dim(self) -> int:
        return self.struct.dim


def _rotary_call(name, params: ksa_params, rotary: Rotary, tensors, outputs, names, stream):
    import torch
    if tensors[0] is None and tensors[1] is None:
        raise ValueError(f"{names[0]} and {names[1]} are both missing")
    if stream is not None and any(x is not None and y is None for x, y in zip(tensors, outputs)):
        if stream.device != rotary.device:
            raise ValueError("stream belongs to another device than the tensors")
        with torch.cuda.stream(stream):      # what is allocated here belongs to `stream`
            return _rotary_call(name, params, rotary, tensors, outputs, names, None)
    (q, k), (q_out, k_out) = tensors, outputs
    batch, n_text, c, m, _, _, n_q_heads, n_kv_heads, d = _FIELDS.unpack_from(params)
    rows = n_text // c * (c + m) + n_text % c if c > 0 else -1
    if q is not None and q_out is None:
        q_out = torch.empty_like(q)
    if k is not None and k_out is None:
        k_out = torch.empty_like(k)
    dev, shapes, plain = rotary._dev, ((batch, rows, n_q_heads, d), (batch, rows, n_kv_heads, d)), True
    for x, y, shape in ((q, q_out, shapes[0]), (k, k_out, shapes[1])):     # as in _plain: in as few steps as possible
        if x is None:
            plain = plain and y is None
        else:
            plain = plain and (x.dtype is torch.bfloat16 and y.dtype is torch.bfloat16 and x.shape == shape and y.shape == shape and x.is_contiguous() and
                               y.is_contiguous() and x.get_device() == dev and y.get_device() == dev)
    strides = (None,) * 4
    if not plain:
        augmented_rows(params, n_text)   # (parameters that make no sense are reported under this name)
        for x, y, what, shape in ((q, q_out, names[0], shapes[0]), (k, k_out, names[1], shapes[1])):
            if x is None:
                if y is not None:
                    raise ValueError(f"an output is given for {what}, which is missing")
                continue
            for t in (x, y):
                _require(t, what, torch.bfloat16, 4)
                if tuple(t.shape) != shape:
                    raise ValueError(f"{what}: expected {shape}, got {tuple(t.shape)}")
                if t.get_device() != dev:
                    raise ValueError(f"{what} lies on another device than the frequencies")
        strides = tuple(_strides_of(t) if t is not None else None for t in (q, k, q_out, k_out))
    _on_device(dev, name, stream, C.byref(params), rotary._arg, *(t.data_ptr() if t is not None else None for t in (q, k, q_out, k_out)), *strides)
    return q_out, k_out


def ksa_rotary_fwd(params: ksa_params, rotary: Rotary, q, k, q_out=None, k_out=None, stream=None):
    """q [B, L, Hq, d], k [B, L, Hkv, d] bf16 of whole augmented sequences -> both turned by their rows' positions (a summary row's is that of its chunk's last
    text).  q or k may be None; an output may be its input.  Gradients: ksa_rotary_bwd."""
    return _rotary_call("ksa_rotary_fwd", params, rotary, (q, k), (q_out, k_out), ("q", "k"), stream)


def ksa_rotary_bwd(params: ksa_params, rotary: Rotary, dq_out, dk_out, dq=None, dk=None, stream=None):
    """Gradients with respect to ksa_rotary_fwd's outputs -> with respect to its q and k."""
    return _rotary_call("ksa_rotary_bwd", params, rotary, (dq_out, dk_out), (dq, dk), ("dq_out", "dk_out"), stream)


def ksa_rotary_step(params: ksa_params, rotary: Rotary, kind: int, q, k, pos, q_out=None, k_out=None, stream=None):
    """The decode loop's new rows, one per sequence: q [B, Hq, d] and k [B, Hkv, d] bf16 (either may be None) turned by pos int32 [B], text indices or summary
    ordinals by `kind` (KSA_ROW_TEXT, KSA_ROW_SUMMARY), before ksa_cache_append and ksa_decode_fwd.  An output may be its input."""
    import torch
    if q is None and k is None:
        raise ValueError("q and k are both missing")
    if stream is not None and (q is not None and q_out is None or k is not None and k_out is None):
        if stream.device != rotary.device:
            raise ValueError("stream belongs to another device than the tensors")
        with torch.cuda.stream(stream):      # what is allocated here belongs to `stream`
            return ksa_rotary_step(params, rotary, kind, q, k, pos, q_out, k_out)
    batch, _, _, _, _, _, n_q_heads, n_kv_heads, d = _FIELDS.unpack_from(params)
    if q is not None and q_out is None:
        q_out = torch.empty_like(q)
    if k is not None and k_out is None:
        k_out = torch.empty_like(k)
    _require(pos, "pos", torch.int32, 1)
    if pos.shape[0] != batch or pos.stride(0) != 1 or pos.get_device() != rotary._dev:
        raise ValueError(f"pos must be {batch} contiguous elements on the frequencies' device")
    strides = []
    for x, y, what, shape in ((q, q_out, "q", (batch, n_q_heads, d)), (k, k_out, "k", (batch, n_kv_heads, d))):
        if x is None and y is not None:
            raise ValueError(f"an output is given for {what}, which is missing")
        for t in (x, y):
            if t is not None:
                _require(t, what, torch.bfloat16, 3)
                if t.shape != shape or t.get_device() != rotary._dev:
                    raise ValueError(f"{what}: expected {shape} on the frequencies' device, got {tuple(t.shape)}")
            strides.append(None if t is None or t.is_contiguous() else _strides_of(t))
    _on_device(rotary._dev, "ksa_rotary_step", stream, C.byref(params), rotary._arg, kind, q.data_ptr() if q is not None else None, k.data_ptr() if k is not None else None,
               pos.data_ptr(), q_out.data_ptr() if q is not None else None, k_out.data_ptr() if k is not None else None, strides[0], strides[2], strides[1], strides[3])
    return q_out, k_out


def ksa_paged_rotary(cache: PagedCache, rotary: Rotary, q, k_new, v_new, cu_rows, start, q_out=None, stream=None):
    """ksa_paged_append of the turned k_new and of v_new [rows, Hkv, d], and q [rows, Hq, d] turned -> q_out, in one launch.  q may be None; q_out may be q.
    What is allocated here belongs to `stream`."""
    import torch
    if stream is not None and q is not None and q_out is None:
        _check_stream(cache, stream)
        with torch.cuda.stream(stream):
            return ksa_paged_rotary(cache, rotary, q, k_new, v_new, cu_rows, start)
    if rotary._dev != cache._dev:
        raise ValueError("the frequencies lie on another device than the cache")
    kv_strides = q_strides = out_strides = None
    if not cache._plain(k_new, v_new, cache._kv, cu_rows, start):
        _rows_of_call(cache, ((k_new, "k_new"), (v_new, "v_new")), cache.params.n_kv_heads, cu_rows, start)
        if not _same_strides(k_new, v_new):
            raise ValueError("k_new and v_new must have the same strides")
        kv_strides = _strides_of(k_new)
    if q is None:
        if q_out is not None:
            raise ValueError("q_out is given, q is missing")
    else:
        plain = q.dtype is torch.bfloat16 and q.shape[1:] == cache._q and q.is_contiguous() and q.get_device() == cache._dev
        if q_out is None:
            q_out = torch.empty_like(q)
        else:
            plain = plain and q_out.dtype is torch.bfloat16 and q_out.shape == q.shape and q_out.is_contiguous() and q_out.get_device() == cache._dev
        if not plain:
            _rows_of_call(cache, ((q, "q"), (q_out, "q_out")), cache.params.n_q_heads, cu_rows, start)
            q_strides, out_strides = _strides_of(q), _strides_of(q_out)
        if q.shape[0] != k_new.shape[0]:
            raise ValueError("q must have as many rows as k_new")
    _paged(cache, "ksa_paged_rotary", stream, rotary._arg, q.data_ptr() if q is not None else None, q_out.data_ptr() if q is not None else None, k_new.data_ptr(),
           v_new.data_ptr(), q_strides, out_strides, kv_strides, cu_rows.data_ptr(), start.data_ptr(), k_new.shape[0])
    return q_out


# ---- a step's rows and pages ----------------------------------------------------------------------------


class PagedStep(NamedTuple):
    """What ksa_paged_advance works out, on the GPU."""
    cu_rows: Any      # int32 [batch + 1]
    start: Any        # int32 [batch]
    lacking: Any      # int32 [1]: columns that got no page
    slots: Any        # int64 [total_rows]: page * page_rows + slot, -1 without a page
    positions: Any    # int32 [total_rows]: rotary positions
    tokens: Any       # int32 [total_rows]: place among the new text tokens, or -1 - s for the s-th summary of its chunk


def paged_advance_workspace_bytes(cache: PagedCache) -> int:
    return int(lib().ksa_paged_advance_workspace_bytes(*cache._args))


def _new_step(cache: PagedCache, total_rows: int) -> PagedStep:
    import torch
    batch = cache._batch[1][0]
    parts = torch.empty(2 * batch + 2 + 2 * total_rows, dtype=torch.int32, device=cache.device).split((batch + 1, batch, 1, total_rows, total_rows))
    return PagedStep(*parts[:3], torch.empty(total_rows, dtype=torch.int64, device=cache.device), *parts[3:])


def ksa_paged_advance(cache: PagedCache, page_refs, held, new_text, total_rows: int, step: Optional[PagedStep] = None, workspace=None, stream=None) -> PagedStep:
    """held, new_text int32 [batch]: text tokens that every sequence holds, and that come (-1: it has ended) -> the step's rows (PagedStep; `step`, one of an
    earlier call, is written again).  The cache's tables and page_refs (int32 [n_pages], table entries that name a page) are brought up to date: columns that nobody sees any
    more are given back, new ones get the lowest free pages.  total_rows: length of the row maps; rows behind the last sequence's get -1, 0 and -1.
    workspace: uint8, at least paged_advance_workspace_bytes(cache) bytes (allocated here if omitted).  What is allocated here belongs to `stream`."""
    import torch
    if stream is not None and (step is None or workspace is None):
        _check_stream(cache, stream)
        with torch.cuda.stream(stream):
            return ksa_paged_advance(cache, page_refs, held, new_text, total_rows, step, workspace)
    if total_rows < 0:
        raise ValueError("total_rows must not be negative")
    i32, dev, (cu_shape, batch), n_pages = torch.int32, cache._dev, cache._batch, cache.struct.n_pages
    if not (page_refs.dtype is i32 and held.dtype is i32 and new_text.dtype is i32 and page_refs.shape == (n_pages,) and held.shape == batch and
            new_text.shape == batch and page_refs.is_contiguous() and held.is_contiguous() and new_text.is_contiguous() and
            page_refs.get_device() == dev and held.get_device() == dev and new_text.get_device() == dev):
        raise ValueError(f"page_refs, held and new_text must be contiguous int32 of {n_pages}, {batch[0]} and {batch[0]} elements on the cache's device")
    if step is None:
        step = _new_step(cache, total_rows)
    else:
        rows = (total_rows,)
        for t, name, dtype, shape in zip(step, PagedStep._fields, (i32, i32, i32, torch.int64, i32, i32), (cu_shape, batch, (1,), rows, rows, rows)):
            if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != dev:
                raise ValueError(f"{name} must be contiguous {dtype} {shape} on the cache's device")
    if workspace is None:
        workspace = torch.empty(paged_advance_workspace_bytes(cache), dtype=torch.uint8, device=cache.device)
    elif workspace.dtype is not torch.uint8 or workspace.get_device() != cache._dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the cache's device")
    _paged(cache, "ksa_paged_advance", stream, page_refs.data_ptr(), held.data_ptr(), new_text.data_ptr(), step.cu_rows.data_ptr(), step.start.data_ptr(),
           step.lacking.data_ptr(), step.slots.data_ptr(), step.positions.data_ptr(), step.tokens.data_ptr(), total_rows, workspace.data_ptr(), workspace.numel())
    return step


def pack_cache(params: ksa_params, k_sum, v_sum, k_txt, v_txt, txt_base: int):
    """Place logical rows into a physical cache pair following ksa_cache_geometry (data movement only).

    k_sum/v_sum [B, Hkv, S, d]: summary ordinal u at index u.  k_txt/v_txt [B, Hkv, W, d]: slot t holds text
    index txt_base + t (slots whose text index is >= n_text are ignored).  Unwritten rows stay zero.
    """
    import torch
    s_cap, rows = cache_geometry(params)
    B, Hkv, S, d = k_sum.shape
    k_cache = torch.zeros((B, Hkv, rows, d), dtype=k_sum.dtype, device=k_sum.device)
    v_cache = torch.zeros_like(k_cache)
    n = min(S, s_cap)
    k_cache[:, :, :n] = k_sum[:, :, :n]
    v_cache[:, :, :n] = v_sum[:, :, :n]
    W = k_txt.shape[2]
    slots = [t for t in range(W) if txt_base + t < params.n_text]
    dst = torch.tensor([cache_text_row(params, txt_base + t) for t in slots], dtype=torch.long, device=k_sum.device)
    src = torch.tensor(slots, dtype=torch.long, device=k_sum.device)
    k_cache[:, :, dst] = k_txt[:, :, src]
    v_cache[:, :, dst] = v_txt[:, :, src]
    return k_cache, v_cache
