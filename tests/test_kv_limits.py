"""Sizes that do not fit one launch (2^32 threads) are refused by the key/value
calls before anything is enqueued."""
import ctypes as C
import os

import pytest
import torch

import paper_2607_05708_amd as pm

pytestmark = pytest.mark.skipif(not os.path.exists(pm.library_path()), reason="libmemattn.so not built")
FAKE = 0x100000  # never dereferenced: the calls are refused, or there is no GPU that could run them
UNSUPPORTED = -2


def kv(heads=8, d=128, fmt=pm.MEM_KV_FP4):
    return pm.MemKv(pm.MemPages(FAKE, 64, pm.mem_kv_page_bytes(64, heads, d, fmt), FAKE, 8, 8), 64, heads, d, fmt)


def move(name, n, dtype, heads=8, d=128):
    rows = [pm.MemKvRows(at, heads * d, d) for at in (1 << 44, 1 << 45)]
    return getattr(pm.lib(), name)(C.byref(kv(heads, d)), C.byref(rows[0]), C.byref(rows[1]), dtype, FAKE, FAKE, n, None)


def attend(m, heads, heads_q, ragged=False, d=64):
    cache = kv(heads, d)
    a = pm.MemAttendArgs(FAKE, FAKE, m, 8, heads_q, FAKE if ragged else None, None, 0.1, 0.0, None, 0, 0, None, None,
                         None)
    need = pm.lib().mem_attend_workspace_bytes(C.byref(cache), m, 8, m, heads_q)
    return pm.lib().mem_attend(C.byref(cache), C.byref(a), FAKE, m, heads_q * d, d, FAKE, FAKE,
                               FAKE if need else None, need, None)


# the first sizes of 2^24 workgroups or more: an item is 8 elements, or 4 of fp32 rows read; 4 items a thread
MOVES = [("mem_kv_write", 1 << 26, pm.MEM_BF16, 8, 128), ("mem_kv_write", 1 << 26, pm.MEM_F32, 8, 128),
         ("mem_kv_read", 1 << 26, pm.MEM_BF16, 8, 128), ("mem_kv_read", 1 << 25, pm.MEM_F32, 8, 128),
         ("mem_kv_read", 1 << 29, pm.MEM_F32, 1, 64), ("mem_kv_write", 1 << 18, pm.MEM_BF16, 1024, 256)]
CALLS = [(1 << 21, 8, 8), (1 << 22, 4, 16), (1 << 24, 1, 1)]


@pytest.mark.parametrize("name,n,dtype,heads,d", MOVES)
def test_moves_beyond_a_launch(name, n, dtype, heads, d):
    assert move(name, n, dtype, heads, d) == UNSUPPORTED
    assert move(name, 2 * n, dtype, heads, d) == UNSUPPORTED
    assert move(name, (1 << 63) - 1, dtype, heads, d) == UNSUPPORTED


@pytest.mark.parametrize("m,heads,heads_q", CALLS)
def test_attention_beyond_a_launch(m, heads, heads_q):
    assert attend(m, heads, heads_q) == UNSUPPORTED
    assert attend(m, heads, heads_q, ragged=True) == UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would run")
def test_sizes_below_are_not_refused():
    # (they end at the launch, for want of a GPU)
    for name, n, dtype, heads, d in MOVES:
        assert move(name, n - 64, dtype, heads, d) not in (0, -1, UNSUPPORTED)
    for m, heads, heads_q in CALLS:
        assert attend(m - 1, heads, heads_q) not in (0, -1, UNSUPPORTED)
