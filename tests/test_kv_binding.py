"""The key/value binding's own checks: what never reaches the library."""
import os

import pytest
import torch

import paper_2607_05708_amd as pm

pytestmark = pytest.mark.skipif(not os.path.exists(pm.library_path()) or torch.cuda.is_available(),
                                reason="library not built, or a GPU there: host tensors stand for device ones here")
WIDE = [2 ** 31, 2 ** 32 + 5, 2 ** 40 + 64, -2 ** 31 - 1]


def host_cache():
    """A cache over host tensors, whose device number (-1) passes for a GPU's; calls end in a device error at most."""
    c = pm.KvCache.__new__(pm.KvCache)
    c._dev, c.pool = -1, torch.zeros((4, pm.mem_kv_page_bytes(32, 1, 64, pm.MEM_KV_FP4)), dtype=torch.uint8)
    c.table = torch.arange(4, dtype=torch.int32).view(2, 2)
    c.page_tokens, c.heads, c.head_dim, c.format = 32, 1, 64, pm.MEM_KV_FP4
    c._c = pm.MemKv(pm.MemPages(c.pool.data_ptr(), 4, c.pool.shape[1], c.table.data_ptr(), 2, 2), 32, 1, 64,
                    pm.MEM_KV_FP4)
    c._ref = pm.C.byref(c._c)
    return c


@pytest.fixture
def on_host(monkeypatch):
    monkeypatch.setattr(pm, "_dev", lambda t, name: t)
    monkeypatch.setattr(pm, "_get_device", lambda: -1)
    monkeypatch.setattr(pm, "_raw_stream", lambda dev: 0)


def attend(cache, **kw):
    q = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    out = torch.zeros((2, 2, 64), dtype=torch.bfloat16), None
    kw = dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8), **kw) if "workspace" not in kw else kw
    return pm.mem_attend(cache, torch.zeros(2, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32), q, 1.0,
                         out=out, **kw)


@pytest.mark.parametrize("x", WIDE)
def test_integers_of_more_than_32_bits_are_refused(on_host, x):
    with pytest.raises(ValueError):
        attend(host_cache(), window=x)
    for i in range(4):
        sizes = [32, 1, 64, pm.MEM_KV_FP4]
        sizes[i] = x
        with pytest.raises(ValueError):
            pm.mem_kv_page_bytes(*sizes)
        with pytest.raises(ValueError):
            pm.KvCache(host_cache().pool, host_cache().table, *sizes)
    for args in ((2, x, 2, 2), (2, 2, 2, x)):
        with pytest.raises(ValueError):
            pm.mem_attend_workspace_bytes(host_cache(), *args)
    with pytest.raises(pm.MemError, match="launch"):         # without a GPU the same call ends there
        attend(host_cache(), window=7)


def test_calls_need_the_caches_gpu_to_be_the_current_one(on_host, monkeypatch):
    x, at = torch.zeros((2, 1, 64)), torch.zeros(2, dtype=torch.int32)
    calls = [lambda: attend(host_cache()), lambda: pm.mem_kv_write(host_cache(), x, x.clone(), at, at),
             lambda: pm.mem_kv_read(host_cache(), at, at, out=(x, x.clone()))]
    for call in calls:
        with pytest.raises(pm.MemError, match="launch"):     # without a GPU the call ends there
            call()
    monkeypatch.setattr(pm, "_get_device", lambda: 3)
    for call in calls:
        with pytest.raises(ValueError, match="current"):
            call()


def test_a_workspace_has_the_memory_that_it_counts(on_host):
    one = torch.zeros(1, dtype=torch.uint8)
    for bad in (one.expand(1 << 20), torch.zeros((1024, 2048), dtype=torch.uint8)[:, ::2]):
        with pytest.raises(ValueError, match="workspace"):
            attend(host_cache(), workspace=bad)
