"""Workspaces of the attention over pages: no more than the split blocks of a call can need, and at most
165 MiB."""
import ctypes
import os

import numpy as np
import pytest

from paper_2606_24467_amd import build as B
from paper_2606_24467_amd import compresskv as C

FAKE = 0x10000000  # aligned, never dereferenced


def _bytes(n_new, hq, hkv, d, dtype=C.BF16, cache=None, max_pages=1 << 14, max_len=0):
    if not os.path.exists(B.lib_path()):
        B.build()
    L = C.lib()
    c = C.CkvPagedCache(batch=len(n_new), n_kv_heads=hkv, head_dim=d, page_size=16, n_pages=9, max_pages=max_pages,
                        dtype=dtype if cache is None else cache, reserved=0, k=FAKE, v=FAKE, k_scale=FAKE,
                        v_scale=FAKE, page_table=FAKE, len=FAKE)
    cu = np.cumsum([0] + list(n_new)).astype(np.int32)
    ch = C.CkvChunk(cu_q=FAKE, cu_q_host=cu.ctypes.data)
    p = C.CkvPagedAttendProblem(n_q_heads=hq, dtype=dtype, max_len=max_len, scale=0.0, q_stride_tok=hq * d,
                                q_stride_head=d)
    return L.compresskv_paged_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(ch), ctypes.byref(p))


def _parts(splits, rows, d):
    """Bytes of the partial results of so many splits of blocks of so many rows."""
    return sum(-(-splits * rows * x // 256) * 256 for x in (8, 4 * d))


@pytest.mark.parametrize("n_new,hq,hkv,d,max_len,splits,rows", [
    # one split more than blocks / the splits' number of workgroups, for each block that may be split
    ((2048,), 32, 8, 128, 32768, 256 + 512, 256),      # 256 blocks, split for 512 workgroups
    ((100,), 32, 8, 128, 8192, 16 * 32, 256),          # 16 blocks, 32 splits of 256 keys at most
    ((20,), 32, 8, 128, 1 << 18, 8 + 1024, 80),        # 8 blocks of 80 rows, for 1024
    ((1,), 32, 8, 128, 1 << 18, 8 + 1024, 4),          # single tokens, for 1024
    ((1,), 32, 8, 128, 1000, 8 * 8, 4),                # 8 splits of 128 keys at most
    ((1,) * 40, 8, 2, 64, 1 << 18, 80 + 1024, 4),
])
def test_no_more_than_the_splits_need(n_new, hq, hkv, d, max_len, splits, rows):
    assert _bytes(n_new, hq, hkv, d, max_len=max_len) == _parts(splits, rows, d)


def test_at_most_165_mib():
    most = 0
    for dtype, cache in ((C.BF16, C.BF16), (C.BF16, C.FP8), (C.F32, C.F32), (C.F32, C.FP8)):
        for hq, hkv in ((32, 8), (128, 128), (256, 1), (16, 16), (1, 1)):
            for n_new in ((1,), (8,) * 60, (600,) * 7, (1,) * 200 + (2048,) * 3, (3, 500) * 200, (90000,), (10,) * 500,
                          (1,) * 255 + (300,) * 255):
                if len(n_new) * hkv <= 65535:
                    n = _bytes(n_new, hq, hkv, 128, dtype, cache, 1 << 20)
                    assert 0 < n <= 165 << 20
                    most = max(most, n)
    assert most > 100 << 20
