"""Python binding of libcompresskv (ctypes; argument marshalling only).

The functions mirror the C ABI in include/compresskv.h,
include/compresskv_offline.h and include/compresskv_cache.h and take torch
tensors for device memory; every computation runs in the HIP library.  There is no
fallback: if the library is missing or fails to load, every call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import re

import numpy as np
import torch

from . import build as _build

OK, INVALID_ARGUMENT, UNSUPPORTED, WORKSPACE_TOO_SMALL, HIP_ERROR = 0, 1, 2, 3, 4
F32, BF16, FP4 = 0, 1, 2
POOL_MAX, POOL_AVG = 0, 1
POOL_THEN_MEAN, MEAN_THEN_POOL = 0, 1
INDEX_PER_GROUP, INDEX_LAYER = 0, 1
SCORE_AUTO, SCORE_TWO_PASS, SCORE_ONE_PASS, SCORE_TWO_LAUNCHES = 0, 1, 2, 3
SPIN_DEFAULT, SPIN_CATCHUP_ALL = -1, -2

_INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
_HEADERS = [os.path.join(_INCLUDE, h) for h in ("compresskv.h", "compresskv_offline.h",
                                                "compresskv_cache.h")]


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
