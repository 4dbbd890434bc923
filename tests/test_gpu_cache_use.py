"""The bounded cache as a program uses it: a compressed prompt loaded into it, then
decoding steps (append, attend, evict); calls captured into graphs, on other
streams, and side by side."""
import sys

import numpy as np
import pytest
import torch

from paper_2606_24467_amd import compresskv as C
from paper_2606_24467_amd import workloads as wl
from tests import cache_helpers as H
from tests import parity_helpers as PH
from tests.test_gpu_cache import _check_attend, _evict_oracle

pytestmark = pytest.mark.gpu


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


def _compressed(gpu, heads=False):
    """A ragged batch compressed: (index, rows, cu_seqlens, group budgets, workload)."""
    w = wl.get("ragged8", batch=2, ragged=(300, 900), n_needle=4)
    x = wl.make_layer(w, 0, seed=3)
    q, k, v, cu = PH.device_tensors(x, gpu)
    p = C.Problem(q, k, v, cu, cu_seqlens_host=x.cu_seqlens)
    if heads:
        budgets = [64 + 16 * g for g in range(w.n_kv_heads)]
        idx, ko, vo, _ = C.compress_layer_heads(p, q, k, v, x.srh_mask, budgets)
        return idx, ko, vo, cu, budgets, w
    idx, ko, vo, _ = C.compress_layer(p, q, k, v, x.srh_mask, 128)
    return idx, ko, vo, cu, None, w


@pytest.mark.parametrize("dtype", [C.FP4, torch.bfloat16], ids=["fp4", "bf16"])
@pytest.mark.parametrize("heads", [False, True], ids=["even", "per-group"])
def test_decoding_after_a_compressed_prompt(gpu, dtype, heads):
    idx, ko, vo, cu, budgets, w = _compressed(gpu, heads)
    b, h, d, hq = w.batch, w.n_kv_heads, w.head_dim, w.n_q_heads
    budget = 128
    cache = C.Cache.empty(b, h, budget + 64, d, dtype, gpu)
    cache.load(ko, vo, idx, cu, group_budgets=budgets)
    n = H.state(cache)["length"]
    assert (n == (np.array(budgets)[None] if heads else budget)).all()
    if dtype != C.FP4 and not heads:
        assert (H.bits(cache.k)[:, :, :budget] == H.bits(ko)).all()
    lens = np.diff(cu.cpu().numpy())
    assert (H.state(cache)["seen"] == lens[:, None]).all()
    g = torch.Generator(device=gpu).manual_seed(5)
    for step in range(6):
        tokens = (1, 1, 3, 1, 40, 1)[step]
        _say("step", step, tokens)
        new = torch.randn((b, tokens, 2, h, d), generator=g, device=gpu).to(torch.bfloat16)
        cache.append(new[:, :, 0], new[:, :, 1])
        n_q = min(tokens, 64 * h // hq)
        q = torch.randn((b, n_q, hq, d), generator=g, device=gpu).to(torch.bfloat16)
        before = H.state(cache)
        out = cache.attend(q, accumulate=True)
        _check_attend(cache, q, before, out, True)
        before = H.state(cache)
        cache.evict(budget, n_sinks=4, n_recent=32)
        got, want = H.state(cache), _evict_oracle(before, budget, 4, 32)
        for name in want:
            assert (got[name] == want[name]).all(), name
        assert (got["length"] <= budget).all() and (got["seen"] == before["seen"]).all()


def _step(cache, q, new, budget, stream=None):
    cache.append(new[:, :, 0], new[:, :, 1], stream=stream)
    out = cache.attend(q, accumulate=True, stream=stream)
    cache.evict(budget, n_sinks=2, n_recent=16, stream=stream)
    return out


def _fresh(gpu, dtype, seed=30):
    cache = H.make_cache(C, dtype, [[200, 190], [5, 200]], 224, 64, gpu, seed, past=10)
    g = torch.Generator(device=gpu).manual_seed(31)
    t = torch.bfloat16 if dtype == C.FP4 else dtype
    q = torch.randn((2, 1, 8, 64), generator=g, device=gpu).to(t)
    new = torch.randn((2, 1, 2, 2, 64), generator=g, device=gpu).to(t)
    return cache, q, new


def _busy(gpu):
    x = torch.randn((1 << 20,), device=gpu)
    assert torch.isfinite(x.sum()).item()
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [C.FP4, torch.bfloat16, torch.float32], ids=["fp4", "bf16", "f32"])
def test_steps_in_a_graph(gpu, dtype):
    """A captured decoding step, replayed, walks the cache on exactly as eager steps do."""
    eager, q, new = _fresh(gpu, dtype)
    graph_cache, q2, new2 = _fresh(gpu, dtype)
    side = torch.cuda.Stream(gpu)
    warm, q3, new3 = _fresh(gpu, dtype)
    with torch.cuda.stream(side):
        _step(warm, q3, new3, 200)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(graph_cache, q2, new2, 200)
    for r in range(4):
        want = _step(eager, q, new, 200)
        _busy(gpu)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert (H.bits(out) == H.bits(want)).all(), r
        a, b = H.state(eager), H.state(graph_cache)
        for name in a:
            assert (a[name] == b[name]).all(), (r, name)
        x = torch.randn(q.shape, device=gpu).to(q.dtype)      # the next step's inputs
        for t in (q, q2):
            t.copy_(x)


def test_window_attention_in_a_graph(gpu):
    g = torch.Generator(device=gpu).manual_seed(32)
    for lq, lk in ((1, 3000), (300, 300)):
        q = torch.randn((lq, 8, 128), generator=g, device=gpu).to(torch.bfloat16)
        k, v = (torch.randn((lk, 2, 128), generator=g, device=gpu).to(torch.bfloat16) for _ in "kv")
        cu_q, cu_k = (torch.tensor([0, n], dtype=torch.int32, device=gpu) for n in (lq, lk))
        p = C.WindowProblem(q, k, v, cu_q, cu_k, window=1000, n_sinks=4)
        C.window_attention(p, q, k, v)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = C.window_attention(p, q, k, v)
        for r in range(3):
            q.normal_(generator=g)
            want = C.window_attention(p, q, k, v)
            _busy(gpu)
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert (H.bits(out) == H.bits(want)).all(), (lq, r)


def test_two_graphs_and_other_streams_side_by_side(gpu):
    """Steps on two caches, on streams of their own and replayed together, do not meet."""
    made = [_fresh(gpu, C.FP4, seed) for seed in (40, 41)]
    alone = [_fresh(gpu, C.FP4, seed) for seed in (40, 41)]
    want = [_step(*alone[i], 200) for i in range(2)]
    want = [_step(*alone[i], 200) for i in range(2)]
    streams = [torch.cuda.Stream(gpu) for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):                                    # first step: given streams
        _step(*made[i], 200, stream=streams[i] if i else streams[i].cuda_stream)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):                                    # second step: two graphs
        gph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gph):
            outs.append(_step(*made[i], 200))
        graphs.append(gph)
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert (H.bits(outs[i]) == H.bits(want[i])).all(), i
        a, b = H.state(made[i][0]), H.state(alone[i][0])
        for name in a:
            assert (a[name] == b[name]).all(), (i, name)


def test_refused_calls_leave_everything(gpu):
    cache, q, new = _fresh(gpu, C.FP4)
    before = H.state(cache)
    with pytest.raises(C.CompressKVError):
        cache.evict(0)
    with pytest.raises(C.CompressKVError):
        cache.attend(q.repeat(1, 17, 1, 1))               # 68 rows per group
    with pytest.raises(ValueError):
        cache.attend(q.half())
    with pytest.raises(ValueError):
        cache.attend(q[:, :, ::2])
    with pytest.raises(ValueError):
        cache.append(new[:, :, 0], new[:, :, 1, :1])
    with pytest.raises(ValueError):
        cache.read(torch.float16)
    with pytest.raises(C.CompressKVError):
        cache.attend(q, ws=torch.empty(128, dtype=torch.uint8, device=gpu), accumulate=True)
    full = H.make_cache(C, torch.float32, [[3]], 8, 64, gpu, 1)
    with pytest.raises(C.CompressKVError):
        full.attend(torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device=gpu))
    torch.cuda.synchronize()
    after = H.state(cache)
    for name in before:
        assert (before[name] == after[name]).all(), name


def test_calls_on_the_default_stream_by_its_handle(gpu):
    """stream=0 is the default stream: a call there sees what was enqueued before it, and what
    is enqueued after sees the call."""
    assert C._enter(gpu, 0)[1] == torch.cuda.default_stream(gpu).cuda_stream == 0
    assert C._stream_object(gpu, torch.cuda.default_stream(gpu).cuda_stream) == torch.cuda.default_stream(gpu)
    side = torch.cuda.Stream(gpu)
    assert C._enter(gpu, side.cuda_stream)[1] == side.cuda_stream
    cache = H.make_cache(C, torch.bfloat16, [[60, 40]], 64, 128, gpu, 70)
    q = torch.randn((1, 1, 8, 128), device=gpu).to(torch.bfloat16)
    want = cache.attend(q, accumulate=True)
    weight = cache.weight.clone()
    cache.weight.zero_()
    got = cache.attend(q, accumulate=True, stream=0)
    received = cache.weight.clone()
    cache.evict(32, n_recent=4, stream=0)
    torch.cuda.synchronize()
    assert (H.bits(got) == H.bits(want)).all()
    live = torch.arange(64, device=gpu) < torch.tensor([[60], [40]], device=gpu)
    assert (received[0][live] <= weight[0][live]).all() and (received[0][live] > 0).all()
    assert (cache.length == 32).all()
