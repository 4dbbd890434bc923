"""Python binding of libcompresskv (ctypes; argument marshalling only).

The functions mirror the C ABI in include/compresskv.h,
include/compresskv_offline.h, include/compresskv_cache.h and
include/compresskv_paged.h and take torch tensors for device memory; every computation runs in the HIP library.  There is no
fallback: if the library is missing or fails to load, every call raises.  No call
records a gradient: outputs do not require one, whatever the inputs do (a rotation's gradient
is its transposed rotation).
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import re
import struct

import numpy as np
import torch

from . import build as _build

OK, INVALID_ARGUMENT, UNSUPPORTED, WORKSPACE_TOO_SMALL, HIP_ERROR = 0, 1, 2, 3, 4
F32, BF16, FP4, FP8 = 0, 1, 2, 3
POOL_MAX, POOL_AVG = 0, 1
POOL_THEN_MEAN, MEAN_THEN_POOL = 0, 1
INDEX_PER_GROUP, INDEX_LAYER = 0, 1
SCORE_AUTO, SCORE_TWO_PASS, SCORE_ONE_PASS, SCORE_TWO_LAUNCHES = 0, 1, 2, 3
SPIN_DEFAULT, SPIN_CATCHUP_ALL = -1, -2
ROTARY_HALF, ROTARY_PAIRS = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BLEND = 0, 1, 2

_INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
_HEADERS = [os.path.join(_INCLUDE, h) for h in ("compresskv.h", "compresskv_offline.h",
                                                "compresskv_cache.h", "compresskv_paged.h")]


class CkvProblem(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("pool_type", ctypes.c_int32),
        ("pool_kernel", ctypes.c_int32),
        ("reduce_order", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("cu_seqlens", ctypes.c_void_p),
        ("cu_seqlens_host", ctypes.c_void_p),
        ("k_stride_tok", ctypes.c_int64),
        ("k_stride_head", ctypes.c_int64),
        ("v_stride_tok", ctypes.c_int64),
        ("v_stride_head", ctypes.c_int64),
        ("index_mode", ctypes.c_int32),
        ("scoring", ctypes.c_int32),
        ("spin_limit", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
    ]


class CkvSrhProblem(ctypes.Structure):
    _fields_ = [
        ("n_samples", ctypes.c_int32),
        ("n_steps", ctypes.c_int32),
        ("n_heads", ctypes.c_int32),
        ("ctx_len", ctypes.c_int32),
        ("spans_host", ctypes.c_void_p),
    ]


class CkvErrorProblem(ctypes.Structure):
    _fields_ = [
        ("n_steps", ctypes.c_int32),
        ("d_model", ctypes.c_int32),
        ("budget", ctypes.c_int32),
        ("eps", ctypes.c_float),
    ]


class CkvCache(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("capacity", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("pos", ctypes.c_void_p),
        ("weight", ctypes.c_void_p),
        ("len", ctypes.c_void_p),
        ("seen", ctypes.c_void_p),
    ]


class CkvAttendProblem(ctypes.Structure):
    _fields_ = [
        ("n_q_heads", ctypes.c_int32),
        ("n_q", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("accumulate", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("reserved", ctypes.c_int32),
    ]


class CkvWindowProblem(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("n_sinks", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("cu_q", ctypes.c_void_p),
        ("cu_q_host", ctypes.c_void_p),
        ("cu_k", ctypes.c_void_p),
        ("cu_k_host", ctypes.c_void_p),
        ("q_stride_tok", ctypes.c_int64),
        ("q_stride_head", ctypes.c_int64),
        ("k_stride_tok", ctypes.c_int64),
        ("k_stride_head", ctypes.c_int64),
        ("v_stride_tok", ctypes.c_int64),
        ("v_stride_head", ctypes.c_int64),
    ]


class CkvRotary(ctypes.Structure):
    _fields_ = [
        ("head_dim", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32),
        ("layout", ctypes.c_int32),
        ("amplitude", ctypes.c_float),
        ("turns", ctypes.c_void_p),
        ("reserved", ctypes.c_int32 * 2),
    ]


class CkvPagedCache(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("n_pages", ctypes.c_int32),
        ("max_pages", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("reserved", ctypes.c_int32),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p),
        ("len", ctypes.c_void_p),
    ]


class CkvChunk(ctypes.Structure):
    _fields_ = [
        ("cu_q", ctypes.c_void_p),
        ("cu_q_host", ctypes.c_void_p),
    ]


class CkvPagedAttendProblem(ctypes.Structure):
    _fields_ = [
        ("n_q_heads", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("max_len", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("q_stride_tok", ctypes.c_int64),
        ("q_stride_head", ctypes.c_int64),
        ("reserved", ctypes.c_int32 * 2),
    ]


_LIB = None


def exported_names() -> list[str]:
    """Function names the public headers declare."""
    text = "".join(open(h).read() for h in _HEADERS)
    return sorted(set(re.findall(r"\b(compresskv_[a-z_]+)\s*\(", text)))


def lib() -> ctypes.CDLL:
    """The loaded library (raises if it has not been built)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = _build.lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"libcompresskv is not built ({path} missing); "
                           "run `python -m paper_2606_24467_amd.build`")
    L = ctypes.CDLL(path)
    vp, sz, i32, u8p = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_void_p
    P = ctypes.POINTER(CkvProblem)
    L.compresskv_workspace_bytes.argtypes = [P, u8p, i32]
    L.compresskv_workspace_bytes.restype = sz
    L.compresskv_score.argtypes = [P, vp, vp, u8p, vp, vp, sz, vp]
    L.compresskv_select.argtypes = [P, vp, i32, vp, vp, sz, vp]
    L.compresskv_gather.argtypes = [P, vp, vp, vp, i32, vp, vp, vp]
    L.compresskv_compress_layer.argtypes = [P, vp, vp, vp, u8p, i32, vp, vp, vp, vp, vp, sz, vp]
    for f in ("compresskv_score", "compresskv_select", "compresskv_gather",
              "compresskv_compress_layer"):
        getattr(L, f).restype = ctypes.c_int
    L.compresskv_compress_layer_noalloc.argtypes = [P, vp, vp, vp, u8p, i32, vp, vp, vp, vp, vp]
    L.compresskv_compress_layer_noalloc.restype = ctypes.c_int
    L.compresskv_layers_workspace_bytes.argtypes = [P, i32, u8p]
    L.compresskv_layers_workspace_bytes.restype = sz
    L.compresskv_score_layers.argtypes = [P, i32, vp, vp, u8p, vp, vp, sz, vp]
    L.compresskv_score_layers.restype = ctypes.c_int
    L.compresskv_compress_layers.argtypes = [P, i32, vp, vp, vp, u8p, vp, vp, vp, vp, vp, vp, sz,
                                             vp]
    L.compresskv_compress_layers.restype = ctypes.c_int
    L.compresskv_scoring_path.argtypes = [P, u8p]
    L.compresskv_scoring_path.restype = ctypes.c_int
    L.compresskv_status_string.argtypes = [ctypes.c_int]
    L.compresskv_status_string.restype = ctypes.c_char_p
    L.compresskv_last_error.argtypes = []
    L.compresskv_last_error.restype = ctypes.c_char_p
    SP = ctypes.POINTER(CkvSrhProblem)
    L.compresskv_srh_scores.argtypes = [SP, vp, vp, vp, vp, vp, vp]
    L.compresskv_srh_scores.restype = ctypes.c_int
    L.compresskv_select_srh.argtypes = [i32, i32, vp, i32, vp, vp]
    L.compresskv_select_srh.restype = ctypes.c_int
    L.compresskv_select_heads.argtypes = [P, vp, vp, vp, vp]
    L.compresskv_gather_heads.argtypes = [P, vp, vp, vp, vp, vp, vp, vp]
    L.compresskv_compress_layer_heads.argtypes = [P, vp, vp, vp, u8p, vp, vp, vp, vp, vp, vp, sz,
                                                  vp]
    for f in ("compresskv_select_heads", "compresskv_gather_heads",
              "compresskv_compress_layer_heads"):
        getattr(L, f).restype = ctypes.c_int
    EP = ctypes.POINTER(CkvErrorProblem)
    L.compresskv_layer_error_workspace_bytes.argtypes = [P, EP]
    L.compresskv_layer_error_workspace_bytes.restype = sz
    L.compresskv_layer_error.argtypes = [P, EP, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.compresskv_layer_error.restype = ctypes.c_int
    L.compresskv_allocate_budgets.argtypes = [i32, vp, ctypes.c_int64, i32, i32, vp]
    L.compresskv_allocate_budgets.restype = ctypes.c_int
    CP, AP = ctypes.POINTER(CkvCache), ctypes.POINTER(CkvAttendProblem)
    WP = ctypes.POINTER(CkvWindowProblem)
    L.compresskv_cache_load.argtypes = [CP, i32, i32, vp, vp, vp, vp, vp, vp]
    L.compresskv_cache_append.argtypes = [CP, i32, i32, vp, vp, vp, vp, vp]
    L.compresskv_cache_read.argtypes = [CP, i32, vp, vp, vp]
    L.compresskv_cache_attend.argtypes = [CP, AP, vp, vp, vp, sz, vp]
    L.compresskv_cache_evict.argtypes = [CP, i32, i32, i32, vp, sz, vp]
    L.compresskv_window_attention.argtypes = [WP, vp, vp, vp, vp, vp, sz, vp]
    for f in ("compresskv_cache_load", "compresskv_cache_append", "compresskv_cache_read",
              "compresskv_cache_attend", "compresskv_cache_evict",
              "compresskv_window_attention"):
        getattr(L, f).restype = ctypes.c_int
    L.compresskv_cache_attend_workspace_bytes.argtypes = [CP, AP]
    L.compresskv_cache_evict_workspace_bytes.argtypes = [CP, i32]
    L.compresskv_window_attention_workspace_bytes.argtypes = [WP]
    for f in ("compresskv_cache_attend_workspace_bytes", "compresskv_cache_evict_workspace_bytes",
              "compresskv_window_attention_workspace_bytes"):
        getattr(L, f).restype = sz
    RP, XP = ctypes.POINTER(CkvRotary), vp   # (rows: the bytes of a ckv_rows)
    GP, HP = ctypes.POINTER(CkvPagedCache), ctypes.POINTER(CkvChunk)
    TP, f64 = ctypes.POINTER(CkvPagedAttendProblem), ctypes.c_double
    L.compresskv_rotary_turns.argtypes = [i32, f64, i32, f64, f64, f64, i32, vp]
    L.compresskv_rotary.argtypes = [RP, i32, i32, i32, vp, i32, XP, XP, i32, XP, XP, vp]
    L.compresskv_paged_append.argtypes = [GP, HP, RP, i32, XP, XP, i32, XP, XP, vp]
    L.compresskv_paged_read.argtypes = [GP, i32, vp, vp, vp, vp, vp]
    L.compresskv_paged_attend.argtypes = [GP, HP, TP, vp, vp, vp, sz, vp]
    for f in ("compresskv_rotary_turns", "compresskv_rotary", "compresskv_paged_append",
              "compresskv_paged_read", "compresskv_paged_attend"):
        getattr(L, f).restype = ctypes.c_int
    L.compresskv_paged_attend_workspace_bytes.argtypes = [GP, HP, TP]
    L.compresskv_paged_attend_workspace_bytes.restype = sz
    _LIB = L
    return L


class CompressKVError(RuntimeError):
    def __init__(self, func: str, status: int):
        L = lib()
        self.status = status
        super().__init__(f"{func}: {L.compresskv_status_string(status).decode()}: "
                         f"{L.compresskv_last_error().decode()}")


def _check(func: str, status: int) -> None:
    if status != OK:
        raise CompressKVError(func, status)


def _ptr(t) -> int:
    if t is None:
        return 0
    if isinstance(t, torch.Tensor):
        return t.data_ptr()
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return int(t)


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}


class Problem:
    """A ckv_problem built from the layer's tensors.

    q_win [batch, W, Hq, D]; k, v [T, Hkv, D] with D contiguous;
    cu_seqlens int32 [batch+1] on the device (host copy taken once here).
    """

    def __init__(self, q_win: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                 cu_seqlens: torch.Tensor, *, cu_seqlens_host=None, pool_kernel: int = 7,
                 pool_type: int = POOL_MAX, reduce_order: int = POOL_THEN_MEAN,
                 scale: float | None = None, index_mode: int = INDEX_PER_GROUP,
                 scoring: int = SCORE_AUTO, spin_limit: int = -1):
        if q_win.dim() != 4 or k.dim() != 3 or v.dim() != 3:
            raise ValueError("q_win must be [batch, W, Hq, D], k and v [T, Hkv, D]")
        if q_win.dtype not in _DTYPES or k.dtype != q_win.dtype or v.dtype != q_win.dtype:
            raise ValueError("q_win, k and v must share one dtype, bfloat16 or float32")
        if not q_win.is_contiguous():
            raise ValueError("q_win must be contiguous")
        if k.stride(2) != 1 or v.stride(2) != 1:
            raise ValueError("the head dimension of k and v must be contiguous")
        if cu_seqlens.dtype != torch.int32:
            raise ValueError("cu_seqlens must be int32")
        batch, W, Hq, D = q_win.shape
        host = (cu_seqlens_host if cu_seqlens_host is not None else cu_seqlens.cpu())
        self._cu_host = np.ascontiguousarray(
            host.numpy() if isinstance(host, torch.Tensor) else np.asarray(host), dtype=np.int32)
        if self._cu_host.shape != (batch + 1,):
            raise ValueError("cu_seqlens must have batch+1 entries")
        self.cu_seqlens = cu_seqlens
        self.batch, self.window, self.n_q_heads, self.head_dim = batch, W, Hq, D
        self.n_kv_heads = k.shape[1]
        self.total_tokens = int(self._cu_host[-1])
        self.c = CkvProblem(
            batch=batch, n_q_heads=Hq, n_kv_heads=self.n_kv_heads, head_dim=D, window=W,
            dtype=_DTYPES[q_win.dtype], pool_type=pool_type, pool_kernel=pool_kernel,
            reduce_order=reduce_order, scale=float(scale) if scale else 0.0,
            cu_seqlens=cu_seqlens.data_ptr(), cu_seqlens_host=self._cu_host.ctypes.data,
            k_stride_tok=k.stride(0), k_stride_head=k.stride(1),
            v_stride_tok=v.stride(0), v_stride_head=v.stride(1), index_mode=index_mode,
            scoring=scoring, spin_limit=spin_limit, reserved=0)

    @property
    def lengths(self) -> np.ndarray:
        return np.diff(self._cu_host)


def _mask(srh_mask) -> np.ndarray:
    m = srh_mask.cpu().numpy() if isinstance(srh_mask, torch.Tensor) else np.asarray(srh_mask)
    return np.ascontiguousarray(m.astype(np.uint8))


# ------------------------------------------------------------ C ABI mirrors
def compresskv_workspace_bytes(p: Problem, srh_mask, budget: int) -> int:
    m = _mask(srh_mask)
    n = lib().compresskv_workspace_bytes(ctypes.byref(p.c), m.ctypes.data, int(budget))
    if n == 0:
        raise CompressKVError("compresskv_workspace_bytes", INVALID_ARGUMENT)
    return int(n)


def compresskv_score(p: Problem, q_win, k, srh_mask, scores, ws, stream=None) -> None:
    m = _mask(srh_mask)
    _check("compresskv_score", lib().compresskv_score(
        ctypes.byref(p.c), _ptr(q_win), _ptr(k), m.ctypes.data, _ptr(scores), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


def compresskv_select(p: Problem, scores, budget: int, idx, ws=None, stream=None) -> None:
    _check("compresskv_select", lib().compresskv_select(
        ctypes.byref(p.c), _ptr(scores), int(budget), _ptr(idx), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


def compresskv_gather(p: Problem, k, v, idx, budget: int, k_out, v_out, stream=None) -> None:
    _check("compresskv_gather", lib().compresskv_gather(
        ctypes.byref(p.c), _ptr(k), _ptr(v), _ptr(idx), int(budget), _ptr(k_out), _ptr(v_out),
        _stream(stream)))


def compresskv_compress_layer(p: Problem, q_win, k, v, srh_mask, budget: int, idx, k_out, v_out,
                              scores_or_null, ws, stream=None) -> None:
    m = _mask(srh_mask)
    _check("compresskv_compress_layer", lib().compresskv_compress_layer(
        ctypes.byref(p.c), _ptr(q_win), _ptr(k), _ptr(v), m.ctypes.data, int(budget), _ptr(idx),
        _ptr(k_out), _ptr(v_out), _ptr(scores_or_null), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


def compresskv_compress_layer_noalloc(p: Problem, q_win, k, v, srh_mask, budget: int, idx, k_out,
                                      v_out, scores_or_null, stream=None) -> None:
    m = _mask(srh_mask)
    _check("compresskv_compress_layer_noalloc", lib().compresskv_compress_layer_noalloc(
        ctypes.byref(p.c), _ptr(q_win), _ptr(k), _ptr(v), m.ctypes.data, int(budget), _ptr(idx),
        _ptr(k_out), _ptr(v_out), _ptr(scores_or_null), _stream(stream)))


def _masks(srh_masks, n_q_heads: int) -> np.ndarray:
    m = (srh_masks.cpu().numpy() if isinstance(srh_masks, torch.Tensor)
         else np.asarray(srh_masks))
    m = np.ascontiguousarray(m.astype(np.uint8))
    if m.ndim != 2 or m.shape[1] != n_q_heads:
        raise ValueError(f"srh_masks must be [n_layers, {n_q_heads}]")
    return m


def _ptr_array(items) -> ctypes.Array:
    """Host array of device pointers (kept alive by the caller for the call)."""
    return (ctypes.c_void_p * len(items))(*[_ptr(t) for t in items])


def _addr(arr) -> int:
    return ctypes.cast(arr, ctypes.c_void_p).value


def compresskv_layers_workspace_bytes(p: Problem, srh_masks) -> int:
    m = _masks(srh_masks, p.n_q_heads)
    n = lib().compresskv_layers_workspace_bytes(ctypes.byref(p.c), m.shape[0], m.ctypes.data)
    if n == 0:
        raise CompressKVError("compresskv_layers_workspace_bytes", INVALID_ARGUMENT)
    return int(n)


def compresskv_score_layers(p: Problem, q_wins, ks, srh_masks, scores, ws, stream=None) -> None:
    m = _masks(srh_masks, p.n_q_heads)
    qa, ka = _ptr_array(q_wins), _ptr_array(ks)
    _check("compresskv_score_layers", lib().compresskv_score_layers(
        ctypes.byref(p.c), m.shape[0], _addr(qa), _addr(ka), m.ctypes.data, _ptr(scores),
        _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)))


def compresskv_compress_layers(p: Problem, q_wins, ks, vs, srh_masks, budgets, idxs, k_outs,
                               v_outs, scores_or_null, ws, stream=None) -> None:
    m = _masks(srh_masks, p.n_q_heads)
    bud = np.ascontiguousarray(np.asarray(budgets, dtype=np.int32))
    arrs = [_ptr_array(x) for x in (q_wins, ks, vs, idxs, k_outs, v_outs)]
    qa, ka, va, ia, koa, voa = (_addr(a) for a in arrs)
    _check("compresskv_compress_layers", lib().compresskv_compress_layers(
        ctypes.byref(p.c), m.shape[0], qa, ka, va, m.ctypes.data, bud.ctypes.data, ia, koa, voa,
        _ptr(scores_or_null), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)))


class LayersCall:
    """compresskv_compress_layers with its arguments marshalled once, for
    callers that run the same stack repeatedly (the benchmark's timed loop)."""

    def __init__(self, p: Problem, q_wins, ks, vs, srh_masks, budgets, idxs, k_outs, v_outs,
                 scores_or_null, ws):
        self.p = p
        self.m = _masks(srh_masks, p.n_q_heads)
        self.bud = np.ascontiguousarray(np.asarray(budgets, dtype=np.int32))
        self.arrs = [_ptr_array(x) for x in (q_wins, ks, vs, idxs, k_outs, v_outs)]
        self.addrs = [_addr(a) for a in self.arrs]
        self.keep = (q_wins, ks, vs, idxs, k_outs, v_outs, scores_or_null, ws)
        self.scores = _ptr(scores_or_null)
        self.ws, self.ws_bytes = _ptr(ws), ws.numel()

    def __call__(self, stream=None) -> None:
        qa, ka, va, ia, koa, voa = self.addrs
        _check("compresskv_compress_layers", lib().compresskv_compress_layers(
            ctypes.byref(self.p.c), self.m.shape[0], qa, ka, va, self.m.ctypes.data,
            self.bud.ctypes.data, ia, koa, voa, self.scores, self.ws, self.ws_bytes,
            _stream(stream)))


def compresskv_scoring_path(p: Problem, srh_mask) -> int:
    """1 = single-pass scoring kernel, 2 = two passes over K."""
    m = _mask(srh_mask)
    r = lib().compresskv_scoring_path(ctypes.byref(p.c), m.ctypes.data)
    if r < 0:
        raise CompressKVError("compresskv_scoring_path", -r)
    return r


# ------------------------------------------------------ tensor conveniences
def workspace(p: Problem, srh_mask, budget: int, device) -> torch.Tensor:
    return torch.empty(compresskv_workspace_bytes(p, srh_mask, budget), dtype=torch.uint8,
                       device=device)


def score(p: Problem, q_win, k, srh_mask, ws=None, stream=None) -> torch.Tensor:
    scores = torch.empty((p.n_kv_heads, p.total_tokens), dtype=torch.float32, device=k.device)
    if ws is None:
        ws = workspace(p, srh_mask, p.window, k.device)
    compresskv_score(p, q_win, k, srh_mask, scores, ws, stream)
    return scores


def select(p: Problem, scores, budget: int, stream=None) -> torch.Tensor:
    idx = torch.empty((p.batch, p.n_kv_heads, budget), dtype=torch.int32, device=scores.device)
    compresskv_select(p, scores, budget, idx, None, stream)
    return idx


def gather(p: Problem, k, v, idx, budget: int, stream=None):
    shape = (p.batch, p.n_kv_heads, budget, p.head_dim)
    k_out = torch.empty(shape, dtype=k.dtype, device=k.device)
    v_out = torch.empty(shape, dtype=v.dtype, device=v.device)
    compresskv_gather(p, k, v, idx, budget, k_out, v_out, stream)
    return k_out, v_out


def compress_layer(p: Problem, q_win, k, v, srh_mask, budget: int, *, want_scores=False,
                   ws=None, stream=None):
    """One layer: returns (idx, k_out, v_out, scores or None)."""
    dev = k.device
    shape = (p.batch, p.n_kv_heads, budget, p.head_dim)
    idx = torch.empty((p.batch, p.n_kv_heads, budget), dtype=torch.int32, device=dev)
    k_out = torch.empty(shape, dtype=k.dtype, device=dev)
    v_out = torch.empty(shape, dtype=v.dtype, device=dev)
    scores = (torch.empty((p.n_kv_heads, p.total_tokens), dtype=torch.float32, device=dev)
              if want_scores else None)
    if ws is None:
        ws = workspace(p, srh_mask, budget, dev)
    compresskv_compress_layer(p, q_win, k, v, srh_mask, budget, idx, k_out, v_out, scores, ws,
                              stream)
    return idx, k_out, v_out, scores


def layers_workspace(p: Problem, srh_masks, device) -> torch.Tensor:
    return torch.empty(compresskv_layers_workspace_bytes(p, srh_masks), dtype=torch.uint8,
                       device=device)


def score_layers(p: Problem, q_wins, ks, srh_masks, ws=None, stream=None) -> torch.Tensor:
    """Scores of every layer: [n_layers, Hkv, T] fp32."""
    dev = ks[0].device
    scores = torch.empty((len(ks), p.n_kv_heads, p.total_tokens), dtype=torch.float32,
                         device=dev)
    if ws is None:
        ws = layers_workspace(p, srh_masks, dev)
    compresskv_score_layers(p, q_wins, ks, srh_masks, scores, ws, stream)
    return scores


def compress_layers(p: Problem, q_wins, ks, vs, srh_masks, budgets, *, want_scores=False,
                    ws=None, stream=None):
    """Every layer in one call: returns (idx list, k_out list, v_out list,
    scores [n_layers, Hkv, T] or None)."""
    dev = ks[0].device
    idxs, k_outs, v_outs = [], [], []
    for k, B in zip(ks, budgets):
        shape = (p.batch, p.n_kv_heads, int(B), p.head_dim)
        idxs.append(torch.empty(shape[:3], dtype=torch.int32, device=dev))
        k_outs.append(torch.empty(shape, dtype=k.dtype, device=dev))
        v_outs.append(torch.empty(shape, dtype=k.dtype, device=dev))
    scores = (torch.empty((len(ks), p.n_kv_heads, p.total_tokens), dtype=torch.float32,
                          device=dev) if want_scores else None)
    if ws is None:
        ws = layers_workspace(p, srh_masks, dev)
    compresskv_compress_layers(p, q_wins, ks, vs, srh_masks, budgets, idxs, k_outs, v_outs,
                               scores, ws, stream)
    return idxs, k_outs, v_outs, scores


def default_scale(head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim)


# ---------------------------------------------------------------------------
# Offline analyses (include/compresskv_offline.h)
# ---------------------------------------------------------------------------
def srh_problem(attn: torch.Tensor, spans_host) -> tuple:
    """ckv_srh_problem for attention weights [S, N, H, L]; returns it with the
    host span array it points to (keep both alive for the call)."""
    S, N, H, Lc = attn.shape
    spans_np = np.ascontiguousarray(np.asarray(spans_host, dtype=np.int32).reshape(S, 2))
    p = CkvSrhProblem(n_samples=S, n_steps=N, n_heads=H, ctx_len=Lc,
                      spans_host=spans_np.ctypes.data)
    return p, spans_np


def compresskv_srh_scores(p: CkvSrhProblem, attn, gen_tokens, ctx_tokens, spans, scores,
                          stream=None) -> None:
    _check("compresskv_srh_scores",
           lib().compresskv_srh_scores(ctypes.byref(p), _ptr(attn), _ptr(gen_tokens),
                                       _ptr(ctx_tokens), _ptr(spans), _ptr(scores),
                                       _stream(stream)))


def compresskv_select_srh(n_layers: int, heads_per_layer: int, scores, top_k: int, srh_mask,
                          stream=None) -> None:
    _check("compresskv_select_srh",
           lib().compresskv_select_srh(n_layers, heads_per_layer, _ptr(scores), top_k,
                                       _ptr(srh_mask), _stream(stream)))


def srh_scores(attn: torch.Tensor, gen_tokens: torch.Tensor, ctx_tokens: torch.Tensor,
               spans_host, stream=None) -> torch.Tensor:
    """Equation 1 for every head: fp32 [H]."""
    if attn.dtype != torch.float32 or not attn.is_contiguous():
        raise ValueError("attn must be a contiguous fp32 tensor [S, N, H, L]")
    p, spans_np = srh_problem(attn, spans_host)
    spans = torch.from_numpy(spans_np).to(attn.device)
    scores = torch.empty(attn.shape[2], dtype=torch.float32, device=attn.device)
    compresskv_srh_scores(p, attn, gen_tokens.to(torch.int32).contiguous(),
                          ctx_tokens.to(torch.int32).contiguous(), spans, scores, stream)
    return scores


def select_srh(scores: torch.Tensor, n_layers: int, top_k: int, stream=None) -> torch.Tensor:
    """Each layer's top_k heads: uint8 mask [n_layers, heads per layer]."""
    hp = scores.numel() // n_layers
    mask = torch.empty((n_layers, hp), dtype=torch.uint8, device=scores.device)
    compresskv_select_srh(n_layers, hp, scores.contiguous(), top_k, mask, stream)
    return mask


def compresskv_layer_error_workspace_bytes(p: Problem, e: CkvErrorProblem) -> int:
    n = lib().compresskv_layer_error_workspace_bytes(ctypes.byref(p.c), ctypes.byref(e))
    if n == 0:
        raise CompressKVError("compresskv_layer_error_workspace_bytes", INVALID_ARGUMENT)
    return n


def compresskv_layer_error(p: Problem, e: CkvErrorProblem, q_dec, k, v, k_out, v_out, w_o, err,
                           ws, stream=None) -> None:
    _check("compresskv_layer_error",
           lib().compresskv_layer_error(ctypes.byref(p.c), ctypes.byref(e), _ptr(q_dec), _ptr(k),
                                        _ptr(v), _ptr(k_out), _ptr(v_out), _ptr(w_o), _ptr(err),
                                        _ptr(ws), ws.numel() * ws.element_size(),
                                        _stream(stream)))


def layer_error(p: Problem, q_dec: torch.Tensor, k, v, k_out: torch.Tensor, v_out, w_o,
                eps: float = 1e-6, stream=None) -> torch.Tensor:
    """Equations 2-4 for one layer: fp32 [1] on the device.  k_out / v_out are
    the compact caches [batch, Hkv, budget, D] of the eviction path."""
    e = CkvErrorProblem(n_steps=q_dec.shape[1], d_model=w_o.shape[0], budget=k_out.shape[2],
                        eps=eps)
    ws = torch.empty(compresskv_layer_error_workspace_bytes(p, e), dtype=torch.uint8,
                     device=q_dec.device)
    err = torch.empty(1, dtype=torch.float32, device=q_dec.device)
    compresskv_layer_error(p, e, q_dec.contiguous(), k, v, k_out.contiguous(), v_out.contiguous(),
                           w_o.contiguous(), err, ws, stream)
    return err


def allocate_budgets(errors, total: int, min_budget: int, max_budget: int) -> np.ndarray:
    """Layer budgets (host): int32 [n_layers]."""
    e = np.ascontiguousarray(np.asarray(errors, dtype=np.float32))
    out = np.zeros(e.shape[0], dtype=np.int32)
    _check("compresskv_allocate_budgets",
           lib().compresskv_allocate_budgets(e.shape[0], e.ctypes.data, int(total), min_budget,
                                             max_budget, out.ctypes.data))
    return out


# ---------------------------------------------------------------------------
# Head-level (per-group) budgets
# ---------------------------------------------------------------------------
def _budgets(group_budgets) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(group_budgets, dtype=np.int32))


def compresskv_select_heads(p: Problem, scores, group_budgets, idx, stream=None) -> None:
    gb = _budgets(group_budgets)
    _check("compresskv_select_heads",
           lib().compresskv_select_heads(ctypes.byref(p.c), _ptr(scores), gb.ctypes.data,
                                         _ptr(idx), _stream(stream)))


def compresskv_gather_heads(p: Problem, k, v, idx, group_budgets, k_out, v_out,
                            stream=None) -> None:
    gb = _budgets(group_budgets)
    _check("compresskv_gather_heads",
           lib().compresskv_gather_heads(ctypes.byref(p.c), _ptr(k), _ptr(v), _ptr(idx),
                                         gb.ctypes.data, _ptr(k_out), _ptr(v_out),
                                         _stream(stream)))


def compress_layer_heads(p: Problem, q_win, k, v, srh_mask, group_budgets, *, want_scores=False,
                         ws=None, stream=None):
    """S1-S6 with per-group budgets: (idx [batch, total], k_out, v_out
    [batch, total, D], scores or None), total = sum of the budgets."""
    gb = _budgets(group_budgets)
    total = int(gb.sum())
    dev = k.device
    idx = torch.empty((p.batch, total), dtype=torch.int32, device=dev)
    k_out = torch.empty((p.batch, total, k.shape[2]), dtype=k.dtype, device=dev)
    v_out = torch.empty((p.batch, total, v.shape[2]), dtype=v.dtype, device=dev)
    scores = (torch.empty((k.shape[1], p.total_tokens), dtype=torch.float32, device=dev)
              if want_scores else None)
    mask = _mask(srh_mask)
    if ws is None:
        ws = workspace(p, mask, int(gb.max()), dev)
    _check("compresskv_compress_layer_heads",
           lib().compresskv_compress_layer_heads(
               ctypes.byref(p.c), _ptr(q_win), _ptr(k), _ptr(v), mask.ctypes.data, gb.ctypes.data,
               _ptr(idx), _ptr(k_out), _ptr(v_out), _ptr(scores), _ptr(ws),
               ws.numel() * ws.element_size(), _stream(stream)))
    return idx, k_out, v_out, scores


# ---------------------------------------------------------------------------
# The bounded cache and the windowed attention (include/compresskv_cache.h)
# ---------------------------------------------------------------------------
_I64x3 = ctypes.c_int64 * 3
_NO_CONTEXT = contextlib.nullcontext()


def _stream_object(device: torch.device, stream) -> torch.cuda.Stream:
    """The stream that the caller names: a Stream, or a raw handle on the tensors' device.  The
    handle 0 is the default stream (ExternalStream takes 0 for "none given" and answers
    with some other stream)."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    handle = int(stream)
    return (torch.cuda.ExternalStream(handle, device=device) if handle
            else torch.cuda.default_stream(device))


def _enter(device: torch.device, stream):
    """(context, stream handle) of a call on the tensors' device: temporaries and outputs
    are allocated on the stream that the call runs on.  (A decoding step makes
    several of these calls: the raw handle is asked for, not a Stream object.)"""
    if stream is None:
        index = device.index
        here = torch.cuda.current_device() == index
        return (_NO_CONTEXT if here else torch.cuda.device(device),
                torch._C._cuda_getCurrentRawStream(index))
    stream = _stream_object(device, stream)
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors are on {device}")
    return torch.cuda.stream(stream), stream.cuda_stream


def _used_on(stream, device: torch.device, *tensors) -> None:
    """Tensors that a call on a stream of the caller's choice reads or writes: their memory is
    not given out again before that stream is done with them."""
    if stream is None:
        return
    stream = _stream_object(device, stream)
    for t in tensors:
        if t is not None and t.numel():
            t.record_stream(stream)


def _check_ws(ws, device: torch.device) -> None:
    if ws is not None and (ws.device != device or not ws.is_contiguous()):
        raise ValueError(f"ws must be contiguous and on {device}")


def _check_tensor(t, name: str, shape, dtype, device) -> None:
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} (got {t.dtype} {tuple(t.shape)})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}")


def _int32(x, name: str) -> int:
    """x for a 32-bit field of the ABI (ctypes keeps the low bits of a longer one)."""
    x = int(x)
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{name} must fit 32 bits (got {x})")
    return x


def _softmax_scale(scale: float | None) -> float:
    """The ABI's scale: 0 selects 1 / sqrt(head_dim), so no given scale may become 0."""
    if not scale:
        return 0.0
    if scale > 0 and ctypes.c_float(scale).value == 0:
        raise ValueError(f"scale is 0 in 32 bits (got {scale})")
    return float(scale)


def _check_on_gpu(device: torch.device) -> None:
    if device.type != "cuda":
        raise ValueError(f"the tensors must be on a GPU (got {device})")


def _row_dtype(dtype: torch.dtype) -> int:
    if dtype not in _DTYPES:
        raise ValueError(f"rows and queries are bfloat16 or float32 (got {dtype})")
    return _DTYPES[dtype]


class Cache:
    """A layer's bounded KV cache (ckv_cache) over caller-owned tensors:

    k, v [batch, Hkv, capacity, D] (bfloat16 or float32), or for a 4-bit cache
    uint8 codes [batch, Hkv, capacity, D / 2] with uint8 scales k_scale, v_scale
    [batch, Hkv, capacity, D / 32]; pos int32 and weight float32 [batch, Hkv,
    capacity]; length and seen int32 [batch, Hkv].  All contiguous, on one GPU.
    """

    def __init__(self, k, v, k_scale, v_scale, pos, weight, length, seen):
        fp4 = k_scale is not None
        if k.dim() != 4:
            raise ValueError("k must have four dimensions")
        b, h, cap, w = k.shape
        dev = k.device
        self.batch, self.n_kv_heads, self.capacity = b, h, cap
        self.head_dim = 2 * w if fp4 else w
        dtype = torch.uint8 if fp4 else k.dtype
        if not fp4:
            _row_dtype(dtype)
        if fp4 != (v_scale is not None):
            raise ValueError("k_scale and v_scale come together (a 4-bit cache) or not at all")
        _check_tensor(k, "k", k.shape, dtype, dev)
        _check_tensor(v, "v", k.shape, dtype, dev)
        if fp4:
            shape = torch.Size((b, h, cap, self.head_dim // 32))
            _check_tensor(k_scale, "k_scale", shape, torch.uint8, dev)
            _check_tensor(v_scale, "v_scale", shape, torch.uint8, dev)
        _check_tensor(pos, "pos", k.shape[:3], torch.int32, dev)
        _check_tensor(weight, "weight", k.shape[:3], torch.float32, dev)
        _check_tensor(length, "length", k.shape[:2], torch.int32, dev)
        _check_tensor(seen, "seen", k.shape[:2], torch.int32, dev)
        _check_on_gpu(dev)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pos, self.weight, self.length, self.seen = pos, weight, length, seen
        self.device, self.dtype = dev, (FP4 if fp4 else _DTYPES[dtype])
        self.c = CkvCache(batch=b, n_kv_heads=h, head_dim=self.head_dim, capacity=cap,
                          dtype=self.dtype, reserved=0, k=_ptr(k), v=_ptr(v),
                          k_scale=_ptr(k_scale), v_scale=_ptr(v_scale), pos=_ptr(pos),
                          weight=_ptr(weight), len=_ptr(length), seen=_ptr(seen))
        self._ref = ctypes.byref(self.c)
        self._attends, self._evict_bytes = {}, {}

    @classmethod
    def empty(cls, batch: int, n_kv_heads: int, capacity: int, head_dim: int, dtype,
              device) -> "Cache":
        """A cache without live slots.  dtype: torch.bfloat16, torch.float32 or FP4 (the
        capacity is then rounded up to a multiple of 32)."""
        fp4 = dtype == FP4
        if fp4:
            capacity = -(-capacity // 32) * 32
        shape = (batch, n_kv_heads, capacity)

        def new(last, t):
            return torch.zeros(shape + last, dtype=t, device=device)
        rows = [new((head_dim // 2,), torch.uint8) if fp4 else new((head_dim,), dtype)
                for _ in range(2)]
        scales = [new((head_dim // 32,), torch.uint8) if fp4 else None for _ in range(2)]
        counts = [torch.zeros(shape[:2], dtype=torch.int32, device=device) for _ in range(2)]
        return cls(*rows, *scales, torch.full(shape, -1, dtype=torch.int32, device=device),
                   new((), torch.float32), *counts)

    def _tensors(self):
        return (self.k, self.v, self.k_scale, self.v_scale, self.pos, self.weight, self.length,
                self.seen)

    def load(self, k_rows, v_rows, idx, cu_seqlens, group_budgets=None, stream=None) -> None:
        """Kept rows of compress_layer (k_out, v_out [batch, Hkv, n, D], idx [batch, Hkv, n]),
        or with group_budgets of compress_layer_heads ([batch, total, D], [batch, total])."""
        b, h, d = self.batch, self.n_kv_heads, self.head_dim
        dtype = _row_dtype(k_rows.dtype)
        gb = None
        if group_budgets is None:
            if idx.dim() != 3:
                raise ValueError("idx must be [batch, Hkv, n]")
            n = idx.shape[2]
            shape = torch.Size((b, h, n))
        else:
            gb = _budgets(group_budgets)
            if gb.shape != (h,):
                raise ValueError("group_budgets must have one entry per KV group")
            n = 0
            shape = torch.Size((b, int(gb.sum())))
        _check_tensor(idx, "idx", shape, torch.int32, self.device)
        _check_tensor(k_rows, "k_rows", shape + (d,), k_rows.dtype, self.device)
        _check_tensor(v_rows, "v_rows", shape + (d,), k_rows.dtype, self.device)
        _check_tensor(cu_seqlens, "cu_seqlens", torch.Size((b + 1,)), torch.int32, self.device)
        ctx, handle = _enter(self.device, stream)
        with ctx:
            _check("compresskv_cache_load", lib().compresskv_cache_load(
                self._ref, dtype, n, _ptr(k_rows), _ptr(v_rows), _ptr(idx), _ptr(gb),
                _ptr(cu_seqlens), handle))
        _used_on(stream, self.device, k_rows, v_rows, idx, cu_seqlens, *self._tensors())

    def append(self, k_new, v_new, stream=None) -> None:
        """New tokens' rows [batch, n, Hkv, D], D contiguous."""
        shape, dtype = k_new.shape, k_new.dtype
        if (len(shape) != 4 or v_new.shape != shape or shape[0] != self.batch
                or shape[2] != self.n_kv_heads or shape[3] != self.head_dim):
            raise ValueError("k_new and v_new must be [batch, n, Hkv, D]")
        if v_new.dtype != dtype:
            raise ValueError("k_new and v_new must share one dtype")
        ks, vs = k_new.stride(), v_new.stride()
        if ks[3] != 1 or vs[3] != 1:
            raise ValueError("the head dimension of k_new and v_new must be contiguous")
        if k_new.device != self.device or v_new.device != self.device:
            raise ValueError(f"k_new and v_new must be on {self.device}")
        ctx, handle = _enter(self.device, stream)
        with ctx:
            _check("compresskv_cache_append", lib().compresskv_cache_append(
                self._ref, _row_dtype(dtype), shape[1], k_new.data_ptr(), _I64x3(*ks[:3]),
                v_new.data_ptr(), _I64x3(*vs[:3]), handle))
        _used_on(stream, self.device, k_new, v_new, *self._tensors())

    def read(self, dtype: torch.dtype | None = None, stream=None):
        """(k, v) [batch, Hkv, capacity, D] as values, zeros past the live slots."""
        if dtype is None:
            dtype = torch.bfloat16 if self.dtype == FP4 else self.k.dtype
        code = _row_dtype(dtype)
        shape = (self.batch, self.n_kv_heads, self.capacity, self.head_dim)
        ctx, handle = _enter(self.device, stream)
        with ctx:
            k = torch.empty(shape, dtype=dtype, device=self.device)
            v = torch.empty(shape, dtype=dtype, device=self.device)
            _check("compresskv_cache_read", lib().compresskv_cache_read(
                self._ref, code, k.data_ptr(), v.data_ptr(), handle))
        _used_on(stream, self.device, *self._tensors())
        return k, v

    def attend(self, q, *, scale: float | None = None, accumulate: bool = False, out=None,
               ws=None, stream=None):
        """Attention of q [batch, n_q, Hq, D] over the live slots; returns out, like q.
        accumulate adds what every slot received to its weight."""
        if q.dim() != 4 or q.shape[0] != self.batch or q.shape[3] != self.head_dim:
            raise ValueError("q must be [batch, n_q, Hq, D]")
        _check_tensor(q, "q", q.shape, q.dtype, self.device)
        if out is not None:
            _check_tensor(out, "out", q.shape, q.dtype, self.device)
        _check_ws(ws, self.device)
        key = (q.shape[1], q.shape[2], q.dtype, bool(accumulate), scale)
        known = self._attends.get(key)
        if known is None:
            a = CkvAttendProblem(n_q_heads=q.shape[2], n_q=q.shape[1], dtype=_row_dtype(q.dtype),
                                 accumulate=int(bool(accumulate)),
                                 scale=_softmax_scale(scale), reserved=0)
            n = lib().compresskv_cache_attend_workspace_bytes(self._ref, ctypes.byref(a))
            if n == 0:   # the call itself says why
                _check("compresskv_cache_attend", lib().compresskv_cache_attend(
                    self._ref, ctypes.byref(a), _ptr(q), _ptr(q), 0, 0, 0))
            known = self._attends[key] = (a, ctypes.byref(a), n)
        ctx, handle = _enter(self.device, stream)
        with ctx:
            if out is None:
                out = torch.empty_like(q)
            if ws is None:
                ws = torch.empty(known[2], dtype=torch.uint8, device=self.device)
            _check("compresskv_cache_attend", lib().compresskv_cache_attend(
                self._ref, known[1], q.data_ptr(), out.data_ptr(), ws.data_ptr(),
                ws.numel() * ws.element_size(), handle))
        _used_on(stream, self.device, q, out, ws, *self._tensors())
        return out

    def evict(self, budget: int, *, n_sinks: int = 0, n_recent: int = 0, ws=None,
              stream=None) -> None:
        """Drops the slots of least weight of every group with more than `budget`."""
        _check_ws(ws, self.device)
        budget, n_sinks = _int32(budget, "budget"), _int32(n_sinks, "n_sinks")
        n_recent = _int32(n_recent, "n_recent")
        n = self._evict_bytes.get(budget)
        if n is None:
            n = lib().compresskv_cache_evict_workspace_bytes(self._ref, budget)
            if n == 0:
                raise CompressKVError("compresskv_cache_evict", INVALID_ARGUMENT)
            self._evict_bytes[budget] = n
        ctx, handle = _enter(self.device, stream)
        with ctx:
            if ws is None:
                ws = torch.empty(n, dtype=torch.uint8, device=self.device)
            _check("compresskv_cache_evict", lib().compresskv_cache_evict(
                self._ref, budget, n_sinks, n_recent, ws.data_ptr(),
                ws.numel() * ws.element_size(), handle))
        _used_on(stream, self.device, ws, *self._tensors())


class WindowProblem:
    """A ckv_window_problem for one batch of sequences (its layers share it):
    q [Tq, Hq, D], k, v [Tk, Hkv, D] with D contiguous and any strides; cu_q, cu_k
    int32 [batch + 1] on the device (host copies taken once here, unless given).
    """

    def __init__(self, q, k, v, cu_q, cu_k, *, window: int, n_sinks: int = 0,
                 scale: float | None = None, cu_q_host=None, cu_k_host=None):
        if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape or q.shape[2] != k.shape[2]:
            raise ValueError("q must be [Tq, Hq, D], k and v [Tk, Hkv, D]")
        if q.dtype not in _DTYPES or k.dtype != q.dtype or v.dtype != q.dtype:
            raise ValueError("q, k and v must share one dtype, bfloat16 or float32")
        if q.stride(2) != 1 or k.stride(2) != 1 or v.stride(2) != 1:
            raise ValueError("the head dimension of q, k and v must be contiguous")
        self._host = []
        for name, cu, host, rows in (("cu_q", cu_q, cu_q_host, q.shape[0]),
                                     ("cu_k", cu_k, cu_k_host, k.shape[0])):
            if cu.dtype != torch.int32 or cu.dim() != 1 or not cu.is_contiguous():
                raise ValueError(f"{name} must be contiguous int32 [batch + 1]")
            host = cu.cpu() if host is None else host
            host = np.ascontiguousarray(host.numpy() if isinstance(host, torch.Tensor)
                                        else np.asarray(host), dtype=np.int32)
            if host.shape != tuple(cu.shape) or host.shape[0] < 2:
                raise ValueError(f"{name} must have batch + 1 entries")
            if int(host[-1]) > rows:
                raise ValueError(f"{name} ends past the last row ({int(host[-1])} of {rows})")
            self._host.append(host)
        if cu_q.shape != cu_k.shape:
            raise ValueError("cu_q and cu_k must have the same number of sequences")
        for t in (k, v, cu_q, cu_k):
            if t.device != q.device:
                raise ValueError("q, k, v, cu_q and cu_k must be on one device")
        self.cu_q, self.cu_k, self.device = cu_q, cu_k, q.device
        self._layout = tuple((t.shape, t.stride(), t.dtype) for t in (q, k, v))
        strides = {f"{n}_stride_{w}": t.stride(i) for n, t in (("q", q), ("k", k), ("v", v))
                   for i, w in enumerate(("tok", "head"))}
        self.c = CkvWindowProblem(
            batch=cu_q.shape[0] - 1, n_q_heads=q.shape[1], n_kv_heads=k.shape[1],
            head_dim=q.shape[2], dtype=_DTYPES[q.dtype], window=_int32(window, "window"),
            n_sinks=_int32(n_sinks, "n_sinks"),
            scale=_softmax_scale(scale), cu_q=_ptr(cu_q),
            cu_q_host=self._host[0].ctypes.data, cu_k=_ptr(cu_k),
            cu_k_host=self._host[1].ctypes.data, **strides)
        self._ref = ctypes.byref(self.c)
        self._ws_bytes = lib().compresskv_window_attention_workspace_bytes(self._ref)
        if self._ws_bytes == 0:   # the call itself says why
            _check("compresskv_window_attention", lib().compresskv_window_attention(
                self._ref, 0, 0, 0, 0, 0, 0, 0))


def window_attention(p: WindowProblem, q, k, v, *, out=None, ws=None, stream=None):
    """Causal attention within p's window and first tokens: out [Tq, Hq, D].  q, k and v
    are laid out as the tensors that p was made from."""
    if tuple((t.shape, t.stride(), t.dtype) for t in (q, k, v)) != p._layout:
        raise ValueError("q, k and v must have the shapes, strides and dtype of the problem")
    for t in (q, k, v):
        if t.device != p.device:
            raise ValueError(f"q, k and v must be on {p.device}")
    _check_on_gpu(p.device)
    if out is not None:
        _check_tensor(out, "out", q.shape, q.dtype, p.device)
    _check_ws(ws, p.device)
    ctx, handle = _enter(p.device, stream)
    with ctx:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=p.device)
        if ws is None:
            ws = torch.empty(p._ws_bytes, dtype=torch.uint8, device=p.device)
        _check("compresskv_window_attention", lib().compresskv_window_attention(
            p._ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ws.data_ptr(),
            ws.numel() * ws.element_size(), handle))
    _used_on(stream, p.device, q, k, v, out, ws, p.cu_q, p.cu_k)
    return out


# ---------------------------------------------------------------------------
# Rotary positions and the paged cache (include/compresskv_paged.h)
# ---------------------------------------------------------------------------
def _offsets(cu, host, name: str):
    """Packed sequences' offsets, checked: the host's copy as an array."""
    if cu.dtype != torch.int32 or cu.dim() != 1 or not cu.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32 [batch + 1]")
    host = cu.cpu() if host is None else host
    host = np.ascontiguousarray(host.numpy() if isinstance(host, torch.Tensor)
                                else np.asarray(host), dtype=np.int32)
    if host.shape != tuple(cu.shape) or host.shape[0] < 2:
        raise ValueError(f"{name} must have batch + 1 entries")
    return host


_ROWS = struct.Struct("Pqq")     # a ckv_rows; its bytes are passed as the pointer to it
_CONTIGUOUS = torch.contiguous_format


def _layout(t):
    """What a call's checks of a tensor go by, its device apart."""
    return None if t is None else (t.shape, t.stride(), t.dtype)


def _remember(plans: dict, key, plan):
    """Keeps what the checks of a layout found (a decoding loop makes the same calls over and
    over), of the last few hundred layouts."""
    if len(plans) >= 256:
        plans.clear()
    plans[key] = plan
    return plan


def _token_strides(t, name: str, head_dim: int, dtype, tokens: int, out: bool = False):
    """Checks rows [>= tokens, H, D] of a call, D contiguous: their (token, head) strides."""
    if t.dim() != 3 or t.shape[2] != head_dim or t.shape[0] < tokens:
        raise ValueError(f"{name} must be [tokens, heads, {head_dim}] with {tokens} tokens at least "
                         f"(got {tuple(t.shape)})")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    tok, head, last = t.stride()
    if last != 1:
        raise ValueError(f"the head dimension of {name} must be contiguous")
    if out and t.shape[0] > 1 and t.shape[1] > 1 and not (
            tok >= t.shape[1] * head or head >= t.shape[0] * tok):
        raise ValueError(f"the rows of {name} must not overlap")
    # (the stride of a dimension of one says nothing)
    return (tok if t.shape[0] > 1 else head_dim * max(1, t.shape[1]),
            head if t.shape[1] > 1 else head_dim)


def _check_out(t, out, name: str) -> None:
    if out is not None and out.shape != t.shape:
        raise ValueError(f"{name} must have the shape {tuple(t.shape)} (got {tuple(out.shape)})")


def _out_strides(t, out, name: str, head_dim: int, dtype, tokens: int):
    """The strides of an output like t: of a new dense tensor, or of the one given."""
    _check_out(t, out, name)
    if out is None:
        return (head_dim * t.shape[1], head_dim)
    return _token_strides(out, name, head_dim, dtype, tokens, out=True)


def _check_devices(index: int, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and t.get_device() != index:
            raise ValueError(f"{name} must be on cuda:{index} (got {t.device})")


class Rotary:
    """A rotation of heads by their tokens' positions (ckv_rotary), with its table on the device.

    rotary_dim: the first dimensions, which turn (all of head_dim unless given); layout: which of
    them turn together (ROTARY_HALF, ROTARY_PAIRS); base, scaling (ROTARY_PLAIN, ROTARY_LINEAR,
    ROTARY_BLEND), factor, low, high, original_len: the frequencies, as
    compresskv_rotary_turns computes them; or inv_freq: radians per position [rotary_dim / 2].
    """

    def __init__(self, head_dim: int, rotary_dim: int | None = None, *, layout: int = ROTARY_HALF,
                 base: float = 10000.0, scaling: int = ROTARY_PLAIN, factor: float = 1.0,
                 low: float = 1.0, high: float = 4.0, original_len: int = 8192,
                 amplitude: float = 1.0, inv_freq=None, device):
        head_dim, layout = _int32(head_dim, "head_dim"), _int32(layout, "layout")
        rotary_dim = head_dim if rotary_dim is None else _int32(rotary_dim, "rotary_dim")
        turns = np.zeros(max(0, rotary_dim // 2), dtype=np.uint64)
        if inv_freq is None or rotary_dim < 16 or rotary_dim > 128 or rotary_dim % 16:
            _check("compresskv_rotary_turns", lib().compresskv_rotary_turns(
                rotary_dim, float(base), _int32(scaling, "scaling"), float(factor), float(low), float(high),
                _int32(original_len, "original_len"), turns.ctypes.data))
        else:
            f = np.asarray(inv_freq.cpu() if isinstance(inv_freq, torch.Tensor) else inv_freq,
                           dtype=np.float64)
            if f.shape != turns.shape or not np.isfinite(f).all():
                raise ValueError(f"inv_freq must be {turns.shape[0]} finite numbers")
            part = f.astype(np.longdouble) / (2 * np.arctan2(np.longdouble(0), np.longdouble(-1)))
            part = np.rint((part - np.floor(part)) * np.longdouble(2.0 ** 64))
            turns[:] = np.where(part >= np.longdouble(2.0 ** 64), 0, part).astype(np.uint64)
        self.head_dim, self.rotary_dim, self.layout = head_dim, rotary_dim, layout
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self.device = self.turns.device
        _check_on_gpu(self.device)
        self._plans = {}
        self.c = CkvRotary(head_dim=head_dim, rotary_dim=rotary_dim, layout=layout,
                           amplitude=float(amplitude), turns=self.turns.data_ptr())
        self._ref = ctypes.byref(self.c)


def rotary(r: Rotary, q, k, pos, *, transposed: bool = False, q_out=None, k_out=None, stream=None):
    """q [T, Hq, D] and k [T, Hkv, D] (either may be None) turned by their tokens' positions pos
    int32 [T]: (q_out, k_out).  transposed: the transposed rotation, which takes
    gradients of outputs to those of inputs.  Outputs may be the inputs themselves."""
    key = (_layout(q), _layout(k), _layout(q_out), _layout(k_out), _layout(pos))
    plan = r._plans.get(key)
    if plan is None:
        plan = _remember(r._plans, key, _plan_rotary(r, q, k, pos, q_out, k_out))
    code, n, sides = plan
    index = r.device.index
    if (pos.get_device() != index or (q is not None and q.get_device() != index)
            or (k is not None and k.get_device() != index)
            or (q_out is not None and q_out.get_device() != index)
            or (k_out is not None and k_out.get_device() != index)):
        _check_devices(index, pos=pos, q=q, k=k, q_out=q_out, k_out=k_out)
    (hq, q_in, q_to), (hk, k_in, k_to) = sides
    q_ref = q_to_ref = k_ref = k_to_ref = None
    ctx, handle = _enter(r.device, stream)
    with ctx:
        if hq:
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=_CONTIGUOUS)
            q_ref = _ROWS.pack(q.data_ptr(), *q_in)
            q_to_ref = _ROWS.pack(q_out.data_ptr(), *q_to)
        if hk:
            if k_out is None:
                k_out = torch.empty_like(k, memory_format=_CONTIGUOUS)
            k_ref = _ROWS.pack(k.data_ptr(), *k_in)
            k_to_ref = _ROWS.pack(k_out.data_ptr(), *k_to)
        status = lib().compresskv_rotary(
            r._ref, code, 1 if transposed else 0, n, pos.data_ptr(), hq, q_ref, q_to_ref, hk, k_ref,
            k_to_ref, handle)
        if status:
            _check("compresskv_rotary", status)
    if stream is not None:
        _used_on(stream, r.device, q, k, pos, r.turns, q_out, k_out)
    return q_out, k_out


def _plan_rotary(r: Rotary, q, k, pos, q_out, k_out):
    """(dtype, tokens, (heads, strides, output's strides) of q and of k)."""
    some = q if q is not None else k
    if some is None:
        raise ValueError("q or k must be given")
    dtype, n = some.dtype, some.shape[0]
    code = _row_dtype(dtype)
    if q is not None and k is not None and k.shape[0] != n:
        raise ValueError("q and k must have the same tokens")
    _check_tensor(pos, "pos", torch.Size((n,)), torch.int32, pos.device)
    sides = []
    for x, out, name in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None:
            if out is not None:
                raise ValueError(f"{name}_out is given without {name}")
            sides.append((0, None, None))
            continue
        strides = _token_strides(x, name, r.head_dim, dtype, n)
        sides.append((x.shape[1], strides,
                      _out_strides(x, out, name + "_out", r.head_dim, dtype, n)))
    return code, n, sides


class Chunk:
    """The new tokens of a step, packed by sequence (ckv_chunk): cu_q int32 [batch + 1] on the
    device (a host copy is taken once here, unless given).  A step's layers share it."""

    def __init__(self, cu_q, *, cu_q_host=None):
        self._host = _offsets(cu_q, cu_q_host, "cu_q").copy()
        self._attends = {}
        self.cu_q, self.device, self.batch = cu_q, cu_q.device, cu_q.shape[0] - 1
        self.index = cu_q.get_device()
        self.tokens = int(self._host[-1])
        self.c = CkvChunk(cu_q=cu_q.data_ptr(), cu_q_host=self._host.ctypes.data)
        self._ref = ctypes.byref(self.c)


class PagedCache:
    """A layer's paged KV cache (ckv_paged_cache) over caller-owned tensors:

    k, v [n_pages, Hkv, page_size, D] (bfloat16 or float32), or for an 8-bit cache uint8
    codes of that shape with uint8 scales k_scale, v_scale [n_pages, Hkv, page_size,
    D / 32]; page_table int32 [batch, max_pages]; length int32 [batch], the tokens of each
    sequence, those of the chunk at hand included.  All contiguous, on one GPU.  The table
    and the lengths are the layers' in common, and only read.
    """

    def __init__(self, k, v, k_scale, v_scale, page_table, length):
        fp8 = k_scale is not None
        if k.dim() != 4:
            raise ValueError("k must have four dimensions")
        n, h, size, d = k.shape
        dev = k.device
        dtype = torch.uint8 if fp8 else k.dtype
        if not fp8:
            _row_dtype(dtype)
        if fp8 != (v_scale is not None):
            raise ValueError("k_scale and v_scale come together (an 8-bit cache) or not at all")
        _check_tensor(k, "k", k.shape, dtype, dev)
        _check_tensor(v, "v", k.shape, dtype, dev)
        if fp8:
            shape = torch.Size((n, h, size, d // 32))
            _check_tensor(k_scale, "k_scale", shape, torch.uint8, dev)
            _check_tensor(v_scale, "v_scale", shape, torch.uint8, dev)
        if page_table.dim() != 2:
            raise ValueError("page_table must be [batch, max_pages]")
        _check_tensor(page_table, "page_table", page_table.shape, torch.int32, dev)
        _check_tensor(length, "length", page_table.shape[:1], torch.int32, dev)
        _check_on_gpu(dev)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.page_table, self.length, self.device = page_table, length, dev
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = n, h, size, d
        self.batch, self.max_pages = page_table.shape
        self.dtype = FP8 if fp8 else _DTYPES[dtype]
        self.c = CkvPagedCache(batch=self.batch, n_kv_heads=h, head_dim=d, page_size=size,
                               n_pages=n, max_pages=self.max_pages, dtype=self.dtype, reserved=0,
                               k=_ptr(k), v=_ptr(v), k_scale=_ptr(k_scale), v_scale=_ptr(v_scale),
                               page_table=_ptr(page_table), len=_ptr(length))
        self._ref = ctypes.byref(self.c)
        self._index = dev.index
        self._appends, self._attends = {}, {}

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, dtype,
              page_table, length) -> "PagedCache":
        """A pool of pages without rows.  dtype: torch.bfloat16, torch.float32 or FP8."""
        fp8 = dtype == FP8
        shape = (n_pages, n_kv_heads, page_size)
        dev = page_table.device

        def new(last, t):
            return torch.zeros(shape + (last,), dtype=t, device=dev)
        rows = [new(head_dim, torch.uint8 if fp8 else dtype) for _ in range(2)]
        scales = [new(head_dim // 32, torch.uint8) if fp8 else None for _ in range(2)]
        return cls(*rows, *scales, page_table, length)

    def _tensors(self):
        return (self.k, self.v, self.k_scale, self.v_scale, self.page_table, self.length)

    def _check_batch(self, chunk: Chunk) -> None:
        if chunk.batch != self.batch:
            raise ValueError(f"the chunk has {chunk.batch} sequences, the cache {self.batch}")

    def append(self, chunk: Chunk, k_new, v_new, *, q=None, rotary: Rotary | None = None, q_out=None,
               stream=None):
        """The chunk's rows [T, Hkv, D], D contiguous, into their pages; with a rotation, K turned
        by its tokens' positions, and q [T, Hq, D] too: returns q turned (q_out, which may be
        q), or None."""
        n, index = chunk.tokens, self._index
        key = (_layout(k_new), _layout(v_new), _layout(q), _layout(q_out), n, chunk.batch,
               rotary is None)
        plan = self._appends.get(key)
        if plan is None:
            plan = _remember(self._appends, key,
                             self._plan_append(chunk, k_new, v_new, q, rotary, q_out))
        code, k_in, v_in, heads, q_in, q_to = plan
        if (k_new.get_device() != index or v_new.get_device() != index or chunk.index != index
                or (rotary is not None and rotary.device.index != index)
                or (q is not None and q.get_device() != index)
                or (q_out is not None and q_out.get_device() != index)):
            _check_devices(index, k_new=k_new, v_new=v_new, chunk=chunk.cu_q, q=q, q_out=q_out,
                           rotary=None if rotary is None else rotary.turns)
        q_ref = q_to_ref = None
        ctx, handle = _enter(self.device, stream)
        with ctx:
            if heads:
                if q_out is None:
                    q_out = torch.empty_like(q, memory_format=_CONTIGUOUS)
                q_ref = _ROWS.pack(q.data_ptr(), *q_in)
                q_to_ref = _ROWS.pack(q_out.data_ptr(), *q_to)
            status = lib().compresskv_paged_append(
                self._ref, chunk._ref, None if rotary is None else rotary._ref, code,
                _ROWS.pack(k_new.data_ptr(), *k_in), _ROWS.pack(v_new.data_ptr(), *v_in), heads,
                q_ref, q_to_ref, handle)
            if status:
                _check("compresskv_paged_append", status)
        if stream is not None:
            _used_on(stream, self.device, k_new, v_new, q, q_out, chunk.cu_q,
                     None if rotary is None else rotary.turns, *self._tensors())
        return q_out

    def _plan_append(self, chunk, k_new, v_new, q, rotary, q_out):
        """(dtype, strides of k_new and v_new, heads, strides of q and q_out)."""
        self._check_batch(chunk)
        dtype, d, n = k_new.dtype, self.head_dim, chunk.tokens
        code = _row_dtype(dtype)
        k_in = _token_strides(k_new, "k_new", d, dtype, n)
        v_in = _token_strides(v_new, "v_new", d, dtype, n)
        if k_new.shape[1] != self.n_kv_heads or v_new.shape[1] != self.n_kv_heads:
            raise ValueError(f"k_new and v_new must have {self.n_kv_heads} heads")
        if q is not None and rotary is None:
            raise ValueError("q is given without a rotation")
        if q is None:
            if q_out is not None:
                raise ValueError("q_out is given without q")
            return code, k_in, v_in, 0, None, None
        q_in = _token_strides(q, "q", d, dtype, n)
        return code, k_in, v_in, q.shape[1], q_in, _out_strides(q, q_out, "q_out", d, dtype, n)

    def read(self, cu_k, *, cu_k_host=None, dtype: torch.dtype | None = None, stream=None):
        """(k, v) [cu_k[-1], Hkv, D]: the first tokens of every sequence, packed as cu_k (int32
        [batch + 1]) says, as values; zeros past the sequence's own."""
        if dtype is None:
            dtype = torch.bfloat16 if self.dtype == FP8 else self.k.dtype
        code = _row_dtype(dtype)
        host = _offsets(cu_k, cu_k_host, "cu_k")
        if host.shape[0] != self.batch + 1:
            raise ValueError("cu_k must have batch + 1 entries")
        if cu_k.device != self.device:
            raise ValueError(f"cu_k must be on {self.device}")
        shape = (max(0, int(host[-1])), self.n_kv_heads, self.head_dim)
        ctx, handle = _enter(self.device, stream)
        with ctx:
            k = torch.empty(shape, dtype=dtype, device=self.device)
            v = torch.empty(shape, dtype=dtype, device=self.device)
            _check("compresskv_paged_read", lib().compresskv_paged_read(
                self._ref, code, cu_k.data_ptr(), host.ctypes.data, k.data_ptr(), v.data_ptr(),
                handle))
        _used_on(stream, self.device, cu_k, *self._tensors())
        return k, v

    def attend(self, chunk: Chunk, q, *, scale: float | None = None, max_len: int | None = None,
               out=None, ws=None, stream=None):
        """Causal attention of the chunk's q [T, Hq, D], D contiguous, over the pages, the chunk's
        own rows among them; returns out [T, Hq, D].  max_len: no sequence is longer (default:
        max_pages * page_size).  ws: a workspace, which calls that follow each other on a stream can
        share; without one each call allocates its own (up to 165 MiB)."""
        index = self._index
        key = (q.shape, q.stride(), q.dtype, chunk.tokens, chunk.batch, scale, max_len)
        known = self._attends.get(key)
        if known is None:
            known = _remember(self._attends, key, self._plan_attend(chunk, q, scale, max_len))
        if q.get_device() != index or chunk.index != index:
            _check_devices(index, q=q, chunk=chunk.cu_q)
        if out is not None:
            _check_tensor(out, "out", q.shape, q.dtype, self.device)
        _check_ws(ws, self.device)
        ctx, handle = _enter(self.device, stream)
        with ctx:
            if out is None:
                out = torch.empty_like(q, memory_format=_CONTIGUOUS)
            if ws is None:
                ws = torch.empty(self._attend_bytes(chunk, known), dtype=torch.uint8,
                                 device=self.device)
            status = lib().compresskv_paged_attend(
                self._ref, chunk._ref, known[1], q.data_ptr(), out.data_ptr(), ws.data_ptr(),
                ws.numel() * ws.element_size(), handle)
            if status:
                _check("compresskv_paged_attend", status)
        if stream is not None:
            _used_on(stream, self.device, q, out, ws, chunk.cu_q, *self._tensors())
        return out

    def _plan_attend(self, chunk, q, scale, max_len):
        """(problem, reference to it, what its workspace depends on but for the chunk)."""
        self._check_batch(chunk)
        tok, head = _token_strides(q, "q", self.head_dim, q.dtype, chunk.tokens)
        p = CkvPagedAttendProblem(n_q_heads=q.shape[1], dtype=_row_dtype(q.dtype),
                                  max_len=0 if max_len is None else _int32(max_len, "max_len"),
                                  scale=_softmax_scale(scale), q_stride_tok=tok, q_stride_head=head)
        return p, ctypes.byref(p), (p.n_q_heads, self.n_kv_heads, self.head_dim, self.dtype, p.dtype,
                                    p.max_len or self.max_pages * self.page_size)

    def _attend_bytes(self, chunk, known) -> int:
        """Bytes of workspace; the chunk remembers them, for the layers that share it."""
        n = chunk._attends.get(known[2])
        if n is None:
            n = lib().compresskv_paged_attend_workspace_bytes(self._ref, chunk._ref, known[1])
            if n == 0:   # the call itself says why
                _check("compresskv_paged_attend", lib().compresskv_paged_attend(
                    self._ref, chunk._ref, known[1], 0, 0, 0, 0, 0))
            _remember(chunk._attends, known[2], n)
        return n
