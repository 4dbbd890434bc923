"""Attention over pages writes no further than the workspace that it asks for, however the lengths lie."""
import sys

import numpy as np
import pytest
import torch

from paper_2606_24467_amd import compresskv as C
from tests import cache_helpers as H
from tests import paged_helpers as PH
from tests.test_gpu_paged import KIND_IDS, KINDS
from tests.test_gpu_paged_long import _pool, _randn

pytestmark = pytest.mark.gpu

LENGTHS = {   # of the sequences, up to 4096 tokens
    "equal": lambda b, n: 4096,
    "one": lambda b, n: 4096 if b == n // 2 else 20,
    "rising": lambda b, n: 4096 * (b + 1) // n,
    "halves": lambda b, n: 4096 if b % 2 else 2000,
    "none": lambda b, n: 0,
}
BATCHES = [(1,), (1,) * 70, (8, 1, 3) * 9, (300,), (20, 1) * 40, (600, 1, 90, 1, 1, 30) * 3]


@pytest.mark.parametrize("n_new", BATCHES, ids=lambda n: f"{n[0]}x{len(n)}")
@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
def test_what_lies_behind_a_workspace_stays(gpu, kind, n_new):
    cache_dtype, dtype = kind
    hq, hkv, d, batch = 8, 2, 64, len(n_new)
    print("workspace", kind, batch, file=sys.stderr, flush=True)
    table = torch.randint(0, 300, (batch, 256), generator=torch.Generator(device=gpu).manual_seed(1), device=gpu,
                          dtype=torch.int32)
    length = torch.zeros(batch, dtype=torch.int32, device=gpu)
    cache = C.PagedCache(*_pool(cache_dtype, 300, hkv, d, gpu, 2), table, length)
    q = _randn((sum(n_new), hq, d), dtype, gpu, 3)
    ch = PH.chunk_of(C, n_new, gpu)
    need = cache._attend_bytes(ch, cache._plan_attend(ch, q, None, None))
    room = torch.full((need + (1 << 22),), 0xA5, dtype=torch.uint8, device=gpu)
    for name, of in LENGTHS.items():
        length.copy_(torch.tensor([of(b, batch) for b in range(batch)]))
        out = cache.attend(ch, q, ws=room[:need])
        assert (room[need:] == 0xA5).all(), name
        assert np.array_equal(H.bits(out), H.bits(cache.attend(ch, q))), name
