"""Which dense rows mem_kv_read takes: any strides whose rows do not overlap."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import paper_2607_05708_amd as pm

pytestmark = pytest.mark.skipif(not os.path.exists(pm.library_path()), reason="libmemattn.so not built")
FAKE, FAR = 0x100000, 1 << 40  # never dereferenced: the calls are refused, or there is no GPU that could run them
INVALID = -1
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the calls that are taken would run")


def read(n, heads, k, v, d=64, dtype=pm.MEM_BF16, call="mem_kv_read"):
    """Status for keys and values given as (offset in elements from one place, token stride, head stride)."""
    cache = pm.MemKv(pm.MemPages(FAKE, 4, pm.mem_kv_page_bytes(32, heads, d, pm.MEM_KV_FP4), FAKE, 2, 2), 32, heads, d,
                     pm.MEM_KV_FP4)
    elem = 4 if dtype == pm.MEM_F32 else 2
    rows = [pm.MemKvRows(FAR + elem * at, ts, hs) for at, ts, hs in (k, v)]
    return getattr(pm.lib(), call)(C.byref(cache), C.byref(rows[0]), C.byref(rows[1]), dtype, FAKE, FAKE, n, None)


AWAY = 1 << 30
OVERLAPS = [
    (4, 3, (0, 64, 64), (AWAY, 192, 64)),            # token t + 1 starts at head 1 of token t
    (4, 3, (AWAY, 192, 64), (0, 128, 64)),
    (4, 3, (0, 96, 64), (AWAY, 192, 64)),
    (4, 3, (0, 64, 192), (AWAY, 192, 64)),           # head-major, one token short
    (4, 3, (0, 0, 64), (AWAY, 192, 64)),             # one token for all
    (4, 3, (0, 192, 0), (AWAY, 192, 64)),
    (1, 3, (0, 64, 63), (AWAY, 192, 64)),
    (5, 4, (0, 160, 128), (AWAY, 256, 64)),          # token 3 at 480, head 1 of token 2 at 448
    (4, 3, (0, 192, 64), (0, 192, 64)),              # keys and values in one place
    (4, 3, (0, 192, 64), (128, 192, 64)),            # values start at the keys' head 2
    (4, 3, (0, 384, 64), (191, 384, 64)),            # one element short of a fused array
    (4, 3, (100, 384, 64), (0, 384, 64)),
    (1, 3, (0, 7, 64), (64, 9, 64)),
]
FREE = [
    (4, 3, (0, 192, 64), (AWAY, 192, 64)),
    (4, 3, (0, 64, 256), (AWAY, 65, 260)),           # head-major
    (4, 3, (0, 384, 64), (192, 384, 64)),            # a fused array: [token, keys and values, head]
    (4, 3, (192, 384, 64), (0, 384, 64)),
    (4, 3, (0, 384, 128), (64, 384, 128)),           # [token, head, keys and values]
    (4, 3, (0, 128, 512), (64, 128, 512)),
    (3, 2, (0, 128, 192), (AWAY, 128, 64)),          # neither tokens nor heads lie together: 0 128 256 192 320 448
    (1, 1, (0, 0, 0), (64, 0, 0)),
    (1, 3, (0, 0, 64), (192, 5, 64)),
    (4, 1, (0, 64, 0), (256, 64, 3)),
]


@pytest.mark.parametrize("n,heads,k,v", OVERLAPS)
def test_overlapping_rows_are_refused(n, heads, k, v):
    for dtype in (pm.MEM_BF16, pm.MEM_F32):
        assert read(n, heads, k, v, dtype=dtype) == INVALID
        assert b"overlap" in pm.lib().mem_last_error()


@needs_no_gpu
@pytest.mark.parametrize("n,heads,k,v", FREE)
def test_other_rows_are_taken(n, heads, k, v):
    for dtype in (pm.MEM_BF16, pm.MEM_F32):
        assert read(n, heads, k, v, dtype=dtype) not in (0, INVALID), pm.lib().mem_last_error()


@needs_no_gpu
def test_against_every_element():
    rng = np.random.default_rng(0)
    refused = 0
    for _ in range(600):
        n, heads = int(rng.integers(1, 5)), int(rng.integers(1, 5))
        ts, hs = (int(x) for x in rng.integers(0, 12, 2) * 32)
        apart = int(rng.integers(-40, 40)) * 32
        i, j = np.meshgrid(np.arange(n), np.arange(heads), indexing="ij")
        at = (i * ts + j * hs).reshape(-1, 1) + np.arange(64)
        both = np.concatenate([at.ravel(), at.ravel() + apart])
        overlap = len(np.unique(both)) < both.size
        assert (read(n, heads, (4096, ts, hs), (4096 + apart, ts, hs)) == INVALID) == overlap, (n, heads, ts, hs, apart)
        refused += overlap
    assert 100 < refused < 590


@pytest.mark.parametrize("call", ["mem_kv_read", "mem_kv_write"])
@pytest.mark.parametrize("stride", [1 << 55, 1 << 60, 1 << 62, (1 << 63) - 1])
def test_strides_that_lead_out_of_memory(call, stride):
    # (a sum that wraps would place the rows beside the pool, or anywhere)
    good = (0, 192, 64)
    for bad in ((0, stride, 64), (0, 192, stride)):
        assert read(5, 5, bad, good, call=call) == INVALID
        assert read(5, 5, good, bad, call=call) == INVALID
