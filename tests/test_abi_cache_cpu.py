"""The entry points of include/compresskv_cache.h without a GPU: every invalid call is
refused on the host before any HIP call, with the reason."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_24467_amd import build as B
from paper_2606_24467_amd import compresskv as C

FAKE = 0x10000000  # aligned, never dereferenced: every call below fails validation first
INV, UNS, SMALL = C.INVALID_ARGUMENT, C.UNSUPPORTED, C.WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(B.lib_path()):
        B.build()
    return C.lib()


def _cache(**kw):
    f = dict(batch=2, n_kv_heads=4, head_dim=128, capacity=96, dtype=C.FP4, reserved=0, k=FAKE,
             v=FAKE, k_scale=FAKE, v_scale=FAKE, pos=FAKE, weight=FAKE, len=FAKE, seen=FAKE)
    f.update(kw)
    return C.CkvCache(**f)


def _attend(**kw):
    f = dict(n_q_heads=8, n_q=1, dtype=C.BF16, accumulate=0, scale=0.0, reserved=0)
    f.update(kw)
    return C.CkvAttendProblem(**f)


def _calls(L, c):
    """Every call on this cache, valid but for the cache."""
    c = ctypes.byref(c) if c is not None else None
    a = _attend()
    s = (ctypes.c_int64 * 3)(512, 512, 128)
    yield L.compresskv_cache_load(c, C.BF16, 8, FAKE, FAKE, FAKE, None, FAKE, None)
    yield L.compresskv_cache_append(c, C.BF16, 1, FAKE, s, FAKE, s, None)
    yield L.compresskv_cache_read(c, C.BF16, FAKE, FAKE, None)
    yield L.compresskv_cache_attend(c, ctypes.byref(a), FAKE, FAKE, FAKE, 1 << 40, None)
    yield L.compresskv_cache_evict(c, 8, 0, 0, FAKE, 1 << 40, None)


BAD_CACHES = [
    (dict(batch=0), INV), (dict(n_kv_heads=0), INV), (dict(capacity=0), INV), (dict(reserved=1), INV),
    (dict(dtype=3), UNS), (dict(dtype=-1), UNS), (dict(head_dim=96), UNS), (dict(n_kv_heads=129), UNS),
    (dict(batch=20000), UNS), (dict(capacity=(1 << 24) + 32), UNS), (dict(capacity=95), UNS),
    (dict(k=0), INV), (dict(v=0), INV), (dict(pos=0), INV), (dict(weight=0), INV), (dict(len=0), INV),
    (dict(seen=0), INV), (dict(k_scale=0), INV), (dict(v_scale=0), INV), (dict(k=FAKE + 8), UNS),
    (dict(v=FAKE + 8), UNS), (dict(pos=FAKE + 4), UNS), (dict(weight=FAKE + 4), UNS),
    (dict(len=FAKE + 2), UNS), (dict(seen=FAKE + 1), UNS), (dict(k_scale=FAKE + 8), UNS),
    (dict(v_scale=FAKE + 4), UNS),
]


@pytest.mark.parametrize("fields,status", BAD_CACHES, ids=lambda x: str(x))
def test_bad_caches(L, fields, status):
    c = _cache(**fields)
    for got in _calls(L, c):
        assert got == status
        assert L.compresskv_last_error()
    assert L.compresskv_cache_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(_attend())) == 0
    assert L.compresskv_cache_evict_workspace_bytes(ctypes.byref(c), 8) == 0


def test_no_cache(L):
    assert list(_calls(L, None)) == [INV] * 5


def test_load_refusals(L):
    def call(c=None, dtype=C.BF16, n=8, k=FAKE, v=FAKE, idx=FAKE, groups=None, cu=FAKE):
        c = c or _cache()
        g = None if groups is None else np.array(groups, dtype=np.int32)
        return L.compresskv_cache_load(ctypes.byref(c), dtype, n, k, v, idx,
                                       None if g is None else g.ctypes.data, cu, None)
    for n in (0, -1, 97):
        assert call(n=n) == INV
    for groups in ([1, 2, 3, 0], [1, 2, 3, 97]):
        assert call(groups=groups) == INV
    for arg in ("k", "v", "idx", "cu"):
        assert call(**{arg: 0}) == INV
        assert call(**{arg: FAKE + 2}) == UNS
    for dtype in (C.FP4, 7):
        assert call(dtype=dtype) == UNS
    assert call(c=_cache(dtype=C.F32)) == UNS           # bf16 rows into an fp32 cache
    big = _cache(n_kv_heads=128, capacity=1 << 24)
    assert call(c=big, n=1 << 24) == UNS


def test_append_refusals(L):
    def call(c=None, dtype=C.BF16, n=1, k=FAKE, v=FAKE, ks=(512, 512, 128), vs=(512, 512, 128)):
        ks, vs = ((ctypes.c_int64 * 3)(*s) if s else None for s in (ks, vs))
        return L.compresskv_cache_append(ctypes.byref(c or _cache()), dtype, n, k, ks, v, vs, None)
    assert call(n=0) == INV and call(k=0) == INV and call(v=0) == INV
    assert call(k=FAKE + 8) == UNS and call(v=FAKE + 8) == UNS
    assert call(ks=None) == INV and call(vs=None) == INV
    for i in range(3):
        s = [512, 512, 128]
        s[i] = -8
        assert call(ks=s) == INV and call(vs=s) == INV
        s[i] = 12
        assert call(ks=s) == UNS and call(vs=s) == UNS
        s[i] = 1 << 41
        assert call(ks=s) == INV
    assert call(dtype=C.FP4) == UNS and call(c=_cache(dtype=C.F32)) == UNS


def test_read_refusals(L):
    def call(c=None, dtype=C.BF16, k=FAKE, v=FAKE):
        return L.compresskv_cache_read(ctypes.byref(c or _cache()), dtype, k, v, None)
    assert call(k=0) == INV and call(v=0) == INV and call(k=FAKE + 8) == UNS
    assert call(dtype=C.FP4) == UNS and call(c=_cache(dtype=C.BF16), dtype=C.F32) == UNS


def test_attend_refusals(L):
    c = _cache()

    def call(c=c, q=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
        return L.compresskv_cache_attend(ctypes.byref(c), ctypes.byref(_attend(**kw)), q, out, ws,
                                         ws_bytes, None)
    assert L.compresskv_cache_attend(ctypes.byref(c), None, FAKE, FAKE, FAKE, 1 << 40, None) == INV
    for kw in (dict(n_q_heads=0), dict(n_q_heads=6), dict(n_q=0), dict(accumulate=2),
               dict(reserved=1), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=0),
               dict(out=0), dict(ws=0)):
        assert call(**kw) == INV, kw
    for kw in (dict(dtype=C.FP4), dict(n_q=33), dict(n_q_heads=260), dict(q=FAKE + 8),
               dict(out=FAKE + 8), dict(ws=FAKE + 128)):
        assert call(**kw) == UNS, kw
    assert call(c=_cache(dtype=C.F32), dtype=C.BF16) == UNS
    a = _attend(accumulate=1)
    n = L.compresskv_cache_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(a))
    assert n > 0 and call(accumulate=1, ws_bytes=n - 1) == SMALL


def test_evict_refusals(L):
    c = _cache()

    def call(budget=8, sinks=0, recent=0, ws=FAKE, ws_bytes=1 << 40):
        return L.compresskv_cache_evict(ctypes.byref(c), budget, sinks, recent, ws, ws_bytes, None)
    for kw in (dict(budget=0), dict(budget=97), dict(sinks=-1), dict(recent=-1), dict(ws=0)):
        assert call(**kw) == INV, kw
    assert call(ws=FAKE + 4) == UNS
    n = L.compresskv_cache_evict_workspace_bytes(ctypes.byref(c), 8)
    assert n > 0 and call(ws_bytes=n - 1) == SMALL
    assert L.compresskv_cache_evict_workspace_bytes(ctypes.byref(c), 97) == 0


def _window(cu_q=(0, 5, 9), cu_k=(0, 5, 40), **kw):
    host = [np.array(x, dtype=np.int32) for x in (cu_q, cu_k)]
    f = dict(batch=2, n_q_heads=8, n_kv_heads=4, head_dim=128, dtype=C.BF16, window=16, n_sinks=4,
             scale=0.0, cu_q=FAKE, cu_q_host=host[0].ctypes.data, cu_k=FAKE,
             cu_k_host=host[1].ctypes.data, q_stride_tok=1024, q_stride_head=128, k_stride_tok=512,
             k_stride_head=128, v_stride_tok=512, v_stride_head=128)
    f.update(kw)
    return C.CkvWindowProblem(**f), host


def test_window_refusals(L):
    def call(q=FAKE, k=FAKE, v=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
        p, keep = _window(**kw)
        return L.compresskv_window_attention(ctypes.byref(p), q, k, v, out, ws, ws_bytes, None)
    assert L.compresskv_window_attention(None, FAKE, FAKE, FAKE, FAKE, FAKE, 0, None) == INV
    for kw in (dict(batch=0), dict(n_kv_heads=0), dict(n_q_heads=0), dict(n_q_heads=6),
               dict(window=0), dict(n_sinks=-1), dict(scale=float("nan")), dict(cu_q=0),
               dict(cu_q_host=0), dict(cu_k=0), dict(cu_k_host=0), dict(cu_q=(1, 5, 9)),
               dict(cu_q=(0, 5, 4)), dict(cu_k=(0, 50, 40)), dict(q=0), dict(k=0), dict(v=0),
               dict(out=0)):
        if isinstance(kw.get("cu_q", 0), tuple) or isinstance(kw.get("cu_k", 0), tuple):
            p, keep = _window(**kw)
            got = L.compresskv_window_attention(ctypes.byref(p), FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                                                None)
        elif "cu_q" in kw or "cu_k" in kw:
            p, keep = _window()
            for n, x in kw.items():
                setattr(p, n, x)
            got = L.compresskv_window_attention(ctypes.byref(p), FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                                                None)
        else:
            got = call(**kw)
        assert got == INV, kw
        assert L.compresskv_last_error()
    for kw in (dict(dtype=C.FP4), dict(head_dim=32), dict(n_kv_heads=129, n_q_heads=129),
               dict(n_q_heads=260), dict(cu_k=(0, 5, (1 << 30) + 1)),
               dict(q=FAKE + 8), dict(k=FAKE + 8), dict(v=FAKE + 8), dict(out=FAKE + 8)):
        assert call(**kw) == UNS, kw
    for name in ("q_stride_tok", "q_stride_head", "k_stride_tok", "k_stride_head", "v_stride_tok",
                 "v_stride_head"):
        assert call(**{name: 127}) == INV, name
        assert call(**{name: 132}) == UNS, name
    p, keep = _window(cu_k=(0, 5, 4000), window=4000)     # split over workgroups
    n = L.compresskv_window_attention_workspace_bytes(ctypes.byref(p))
    assert n > 256
    for ws, size, want in ((0, n, INV), (FAKE + 8, n, UNS), (FAKE, n - 1, SMALL)):
        assert L.compresskv_window_attention(ctypes.byref(p), FAKE, FAKE, FAKE, FAKE, ws, size,
                                             None) == want


# ------------------------------------------------------------- the binding
def _tensors(**kw):
    s = (2, 4, 96)
    t = dict(k=torch.zeros(s + (64,), dtype=torch.uint8), v=torch.zeros(s + (64,), dtype=torch.uint8),
             k_scale=torch.zeros(s + (4,), dtype=torch.uint8),
             v_scale=torch.zeros(s + (4,), dtype=torch.uint8),
             pos=torch.zeros(s, dtype=torch.int32), weight=torch.zeros(s),
             length=torch.zeros(s[:2], dtype=torch.int32), seen=torch.zeros(s[:2], dtype=torch.int32))
    t.update(kw)
    return t


@pytest.mark.parametrize("bad", [
    dict(k=torch.zeros(4)), dict(v=torch.zeros(2, 4, 96, 64)), dict(v_scale=None),
    dict(k_scale=torch.zeros(2, 4, 96, 8, dtype=torch.uint8)), dict(pos=torch.zeros(2, 4, 96)),
    dict(weight=torch.zeros(2, 4, 95)), dict(length=torch.zeros(8, dtype=torch.int32)),
    dict(seen=torch.zeros(2, 4, dtype=torch.int64)),
    dict(weight=torch.zeros(2, 4, 192)[:, :, ::2]),
    dict(k_scale=None, v_scale=None)], ids=lambda d: "-".join(d))
def test_binding_refuses_tensors(bad):
    with pytest.raises(ValueError):
        C.Cache(**_tensors(**bad))


def test_binding_refuses_the_host():
    with pytest.raises(ValueError, match="GPU"):
        C.Cache(**_tensors())
    with pytest.raises(ValueError, match="GPU"):
        C.Cache.empty(1, 1, 32, 64, torch.bfloat16, "cpu")
    q, kv = torch.zeros(9, 8, 64), torch.zeros(9, 2, 64)
    cu = torch.tensor([0, 9], dtype=torch.int32)
    p = C.WindowProblem(q, kv, kv, cu, cu, window=4)
    with pytest.raises(ValueError, match="GPU"):
        C.window_attention(p, q, kv, kv)


def test_binding_refuses_window_problems():
    q, kv = torch.zeros(9, 8, 64), torch.zeros(9, 2, 64)
    cu = torch.tensor([0, 9], dtype=torch.int32)
    ok = dict(q=q, k=kv, v=kv, cu_q=cu, cu_k=cu, window=4)
    for bad in (dict(q=q[0]), dict(v=kv[:8]), dict(k=kv.bfloat16()), dict(q=q.half()),
                dict(q=torch.zeros(9, 8, 128)[:, :, ::2]), dict(cu_q=cu.long()), dict(cu_q=cu[:1]),
                dict(cu_k=torch.tensor([0, 3, 9], dtype=torch.int32)),
                dict(cu_q=torch.tensor([0, 10], dtype=torch.int32))):
        with pytest.raises(ValueError):
            C.WindowProblem(**{**ok, **bad})
    for bad in (dict(window=0), dict(n_sinks=-1), dict(q=torch.zeros(9, 7, 64))):
        with pytest.raises(C.CompressKVError):
            C.WindowProblem(**{**ok, **bad})
    p = C.WindowProblem(**ok)
    with pytest.raises(ValueError, match="strides"):
        C.window_attention(p, torch.zeros(9, 16, 64)[:, ::2], kv, kv)


def test_window_without_queries_needs_no_pointers(L):
    p, keep = _window(cu_q=(0, 0, 0))
    assert L.compresskv_window_attention(ctypes.byref(p), None, None, None, None, None, 0, None) == 0
    p, keep = _window(cu_k=(0, 0, 0))                     # without keys: q and out still
    assert L.compresskv_window_attention(ctypes.byref(p), FAKE, None, None, None, FAKE, 1 << 40, None) == INV
    assert L.compresskv_window_attention(ctypes.byref(p), None, None, None, FAKE, FAKE, 1 << 40, None) == INV


def test_the_handle_0_is_the_default_stream(monkeypatch):
    """A raw handle may be 0 (the default stream's).  ExternalStream(0) is some other stream:
    work there is in no order with what the caller has enqueued."""
    device = torch.device("cuda", 0)
    asked = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, device: asked.append(h) or f"handle {h}")
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d: f"default of {d}")
    assert C._stream_object(device, 0) == C._stream_object(device, np.int64(0)) == "default of cuda:0"
    assert not asked
    assert C._stream_object(device, 0x1234) == "handle 4660"


def test_integers_past_32_bits_are_refused():
    """ctypes would keep their low bits: a window of 2^32 + 5 keys would be one of 5."""
    q, kv = torch.zeros(9, 8, 64), torch.zeros(9, 2, 64)
    cu = torch.tensor([0, 9], dtype=torch.int32)
    for bad in (dict(window=(1 << 32) + 5), dict(window=1 << 31), dict(window=4, n_sinks=1 << 32),
                dict(window=-(1 << 32) + 3)):
        with pytest.raises(ValueError, match="32 bits"):
            C.WindowProblem(q, kv, kv, cu, cu, **bad)
    assert C.WindowProblem(q, kv, kv, cu, cu, window=(1 << 31) - 1).c.window == (1 << 31) - 1
    cache = C.Cache.__new__(C.Cache)                      # (a cache itself needs a GPU)
    cache.device = torch.device("cuda", 0)
    for budget, kw in (((1 << 32) + 8, {}), (8, dict(n_sinks=(1 << 32) + 1)), (8, dict(n_recent=1 << 33))):
        with pytest.raises(ValueError, match="32 bits"):
            cache.evict(budget, **kw)


def test_scales_that_32_bits_do_not_hold_are_refused(L):
    """Times log2(e) a scale of 3e38 is infinite, and every zero logit would be NaN; one of 1e-50
    would be 0, which selects the default."""
    for scale, ok in ((3e38, False), (2.3e38, True), (1e-45, True), (-3e38, True), (float("inf"), False)):
        p, keep = _window(scale=scale)
        assert (L.compresskv_window_attention_workspace_bytes(ctypes.byref(p)) > 0) == ok, scale
        n = L.compresskv_cache_attend_workspace_bytes(ctypes.byref(_cache()), ctypes.byref(_attend(scale=scale)))
        assert (n > 0) == ok, scale
        if not ok:
            assert b"scale" in L.compresskv_last_error()
    q, kv = torch.zeros(9, 8, 64), torch.zeros(9, 2, 64)
    cu = torch.tensor([0, 9], dtype=torch.int32)
    with pytest.raises(ValueError, match="scale"):
        C.WindowProblem(q, kv, kv, cu, cu, window=4, scale=1e-50)
    assert C.WindowProblem(q, kv, kv, cu, cu, window=4, scale=0.0).c.scale == 0
    assert C.WindowProblem(q, kv, kv, cu, cu, window=4, scale=1e-45).c.scale > 0


def _window_bytes(L, spans, hq=32, hkv=8, dtype=C.BF16, **kw):
    """Workspace of dense sequences of (queries, keys); 0: refused."""
    cu = [tuple(int(x) for x in np.cumsum([0] + [s[i] for s in spans])) for i in (0, 1)]
    p, keep = _window(cu_q=cu[0], cu_k=cu[1], batch=len(spans), n_q_heads=hq, n_kv_heads=hkv, dtype=dtype,
                      window=1024, **kw)
    return L.compresskv_window_attention_workspace_bytes(ctypes.byref(p))


def test_windows_of_sequences_of_very_different_lengths_are_taken(L):
    """The limit counts the row blocks that there are, not the longest sequence's for every group."""
    assert _window_bytes(L, [(1, 1)] * 300 + [(131072, 131072)]) == 256
    assert _window_bytes(L, [(1, 1)] * 1000 + [(40000, 40000)]) == 256
    assert _window_bytes(L, [(1, 1)] * 65 + [(131072, 131072)], dtype=C.F32) == 256
    assert _window_bytes(L, [(1, 1)] * 4000 + [(1 << 20, 1 << 20)], dtype=C.F32) == 256
    assert _window_bytes(L, [(1 << 30, 1 << 30)], hq=1, hkv=1) == 256
    assert _window_bytes(L, [(1 << 30, 1 << 30)], hq=2, hkv=2) == 0
    assert b"rows" in L.compresskv_last_error()


@pytest.mark.parametrize("dtype", [C.BF16, C.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("apart", [512, 1 << 24], ids=["near", "far"])
def test_windows_of_sequences_without_queries_cost_no_workspace(L, dtype, apart):
    """A chunk split over workgroups needs the same workspace alone and among empty sequences."""
    kw = dict(dtype=dtype, k_stride_tok=apart)
    alone = _window_bytes(L, [(64, 4096)], **kw)
    assert alone > 256
    assert _window_bytes(L, [(0, 0)] * 255 + [(64, 4096)], **kw) == alone
    assert _window_bytes(L, [(0, 50)] * 8000 + [(64, 4096)] + [(0, 0)] * 100, **kw) == alone
