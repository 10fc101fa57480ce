"""The key/value calls without a GPU: declarations, sizes, refusals before any
launch, and the 64-bit model's own pins."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2607_05708_amd as pm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "memattn_kv.h")
FAKE = 0x100000  # never dereferenced: every call below fails validation first

needs_lib = pytest.mark.skipif(not os.path.exists(pm.library_path()), reason="libmemattn.so not built")


def declared_functions():
    text = open(HEADER).read()
    return sorted(set(re.findall(r"MEMATTN_API\s+[\w\s\*]+?\b(mem_\w+)\s*\(", text)))


def test_header_declares_the_calls():
    assert declared_functions() == ["mem_attend", "mem_attend_workspace_bytes", "mem_kv_page_bytes", "mem_kv_read",
                                    "mem_kv_write"]


@needs_lib
def test_library_exports_every_declared_symbol():
    L = C.CDLL(pm.library_path())
    for name in declared_functions():
        assert hasattr(L, name), name


@needs_lib
def test_page_bytes():
    for fmt, t, h, d in ((0, 64, 8, 128), (1, 32, 1, 64), (2, 256, 3, 256), (2, 32, 1, 64)):
        assert pm.mem_kv_page_bytes(t, h, d, fmt) == ref.page_bytes(fmt, t, h, d)
        assert pm.mem_kv_page_bytes(t, h, d, fmt) % 16 == 0
    for bad in ((64, 8, 128, 3), (64, 8, 128, -1), (64, 8, 96, 2), (48, 8, 128, 2), (0, 8, 128, 2),
                (8192, 8, 128, 2), (64, 0, 128, 2), (64, 1025, 128, 2)):
        assert pm.mem_kv_page_bytes(*bad) == 0


def _kv(**kw):
    a = dict(pool=FAKE, n_pages=64, page_bytes=69632, table=FAKE, n_chunks=8, ppc=8, page_tokens=64, heads=8,
             head_dim=128, format=pm.MEM_KV_FP4)
    a.update(kw)
    return pm.MemKv(pm.MemPages(a["pool"], a["n_pages"], a["page_bytes"], a["table"], a["n_chunks"], a["ppc"]),
                    a["page_tokens"], a["heads"], a["head_dim"], a["format"])


BAD_KV = [(dict(format=3), -1), (dict(format=-1), -1), (dict(page_tokens=48), -1), (dict(page_tokens=0), -1),
          (dict(page_tokens=4128), -1), (dict(heads=0), -1), (dict(heads=1025), -1), (dict(head_dim=0), -1),
          (dict(head_dim=96), -2), (dict(head_dim=512), -2), (dict(ppc=0), -1), (dict(ppc=65), -1),
          (dict(n_pages=-1), -1), (dict(n_chunks=-1), -1), (dict(n_pages=1 << 31), -2), (dict(n_chunks=1 << 31), -2),
          (dict(page_bytes=69616), -1), (dict(page_bytes=69640), -1), (dict(page_bytes=0), -1),
          (dict(pool=None), -1), (dict(table=None), -1), (dict(pool=FAKE + 8), -1), (dict(table=FAKE + 2), -1)]


def _rows(**kw):
    a = dict(data=FAKE, ts=1024, hs=128)
    a.update(kw)
    return pm.MemKvRows(a["data"], a["ts"], a["hs"])


@needs_lib
@pytest.mark.parametrize("call", ["mem_kv_write", "mem_kv_read"])
def test_move_refusals(call):
    f = getattr(pm.lib(), call)

    def go(kv=_kv(), k=_rows(), v=_rows(), dtype=pm.MEM_BF16, chunk=FAKE, pos=FAKE, n=4):
        ref_ = lambda x: C.byref(x) if x is not None else None  # noqa: E731
        return f(ref_(kv), ref_(k), ref_(v), dtype, chunk, pos, n, None)

    for kw, status in BAD_KV:
        assert go(kv=_kv(**kw)) == status, kw
        assert pm.lib().mem_last_error()
    assert go(kv=None) == -1
    assert go(k=None) == -1 and go(v=None) == -1
    assert go(k=_rows(data=None)) == -1 and go(v=_rows(data=FAKE + 1)) == -1
    assert go(k=_rows(ts=-1)) == -1 and go(v=_rows(hs=-1)) == -1
    assert go(dtype=2) == -1 and go(chunk=None) == -1 and go(pos=None) == -1 and go(pos=FAKE + 1) == -1
    assert go(n=-1) == -1 and go(n=1 << 40) == -2
    assert go(n=0) == 0
    if call == "mem_kv_read":
        far = 0x10000000
        assert go(k=_rows(data=far, hs=64), v=_rows(data=2 * far)) == -1
        assert go(k=_rows(data=far), v=_rows(data=2 * far, ts=64)) == -1
        assert go(k=_rows(data=FAKE + 4096), v=_rows(data=far)) == -1
        assert b"overlaps" in pm.lib().mem_last_error()


@needs_lib
def test_attend_refusals():
    L = pm.lib()

    def go(kv=_kv(), q=FAKE, total_q=4, ts=4096, hs=128, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40, args=True, **kw):
        a = dict(tok_len=FAKE, ids=FAKE, m=4, k=8, heads_q=32, q_offsets=None, q_pos=None, scale=0.1, softcap=0.0,
                 slopes=None, causal=0, window=0, prefix_len=None, chunk_ns=None, query_ns=None)
        a.update(kw)
        arg = pm.MemAttendArgs(*a.values())
        return L.mem_attend(C.byref(kv) if kv is not None else None, C.byref(arg) if args else None, q, total_q, ts,
                            hs, out, lse, ws, ws_bytes, None)

    for kw, status in BAD_KV:
        assert go(kv=_kv(**kw)) == status, kw
    inf, nan = float("inf"), float("nan")
    for kw in (dict(kv=None), dict(args=False), dict(m=-1), dict(total_q=-1), dict(k=0), dict(k=4097),
               dict(heads_q=0), dict(heads_q=33), dict(heads_q=2048), dict(scale=0.0), dict(scale=nan),
               dict(scale=inf), dict(scale=-1.0), dict(softcap=-1.0), dict(softcap=inf), dict(softcap=nan),
               dict(window=-1), dict(m=0), dict(m=3), dict(ids=None), dict(tok_len=None), dict(chunk_ns=FAKE),
               dict(q=None), dict(out=None), dict(q=FAKE + 1), dict(out=FAKE + 8), dict(ids=FAKE + 2),
               dict(slopes=FAKE + 1), dict(lse=FAKE + 2), dict(ts=-1), dict(hs=-1)):
        assert go(**kw) == -1, kw
        assert L.mem_last_error()
    assert go(total_q=1 << 26, m=1 << 26) == -2
    assert go(total_q=0) == 0 and go(total_q=0, m=0) == 0


@needs_lib
def test_attend_workspace():
    L = pm.lib()
    size = lambda kv, m, k, n, hq: L.mem_attend_workspace_bytes(C.byref(kv), m, k, n, hq)  # noqa: E731
    for bad in ((_kv(format=9), 4, 8, 4, 32), (_kv(), -1, 8, 4, 32), (_kv(), 4, 0, 4, 32), (_kv(), 4, 8, -1, 32),
                (_kv(), 4, 8, 4, 31), (_kv(), 0, 8, 0, 32)):
        assert size(*bad) == 0
    assert size(_kv(), 4, 4096, 4, 32) < 1 << 30


@needs_lib
@pytest.mark.parametrize("total_q", [(1 << 30) // 32 + 1, 1 << 58, (1 << 63) - 1])
def test_attend_refuses_more_rows_than_it_can_number(total_q):
    L, kv = pm.lib(), _kv()
    a = pm.MemAttendArgs(FAKE, FAKE, 1, 8, 32, None, None, 0.1, 0.0, None, 0, 0, None, None, None)
    assert L.mem_attend(C.byref(kv), C.byref(a), FAKE, total_q, 4096, 128, FAKE, FAKE, FAKE, 1 << 40, None) == -2
    assert L.mem_attend_workspace_bytes(C.byref(kv), 1, 8, total_q, 32) == 0


def test_binding_refuses_host_tensors():
    cpu = torch.zeros((4, 69632), dtype=torch.uint8)
    with pytest.raises(ValueError):
        pm.KvCache(cpu, torch.zeros((1, 4), dtype=torch.int32), 64, 8, 128, pm.MEM_KV_FP4)


# ---------------------------------------------------------------- the model itself

def test_model_values_of_codes():
    assert ref.GRID[ref.FP8][-1] == 448 and ref.GRID[ref.FP8][1] == 2.0 ** -9 and len(ref.GRID[ref.FP8]) == 127
    x = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(x, ref.GRID[ref.FP8])


def test_model_scales():
    for fmt, top in ((ref.FP4, 7.0), (ref.FP8, 464.0)):
        assert ref.scale_exponent(fmt, top) == 0
        assert ref.scale_exponent(fmt, np.nextafter(top, 1e9)) == 1
        assert ref.scale_exponent(fmt, top / 2) == -1
        assert ref.scale_exponent(fmt, 0.0) == -110 and ref.scale_exponent(fmt, 1e-40) == -110


def test_model_rounding_is_within_half_a_step():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64))
    for fmt in (ref.FP4, ref.FP8):
        codes, scale = ref.encode_rows(fmt, x)
        y = ref.decode_rows(fmt, codes, scale)
        s = np.repeat(2.0 ** (scale.astype(float) - 127), 32, -1)
        grid = ref.GRID[fmt]
        step = np.diff(grid)[np.clip(np.searchsorted(grid, np.abs(x) / s) - 1, 0, len(grid) - 2)] * s
        assert np.all(np.abs(x - y) <= step / 2 + 1e-15)
        again = ref.decode_rows(fmt, *ref.encode_rows(fmt, y))
        assert np.array_equal(again, y) or fmt == ref.FP4   # FP4: 6 * 2^e may take the next finer scale's 6
    t = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)
    assert np.array_equal(ref.to_bf16(x.astype(np.float32)), t.double().numpy())


def test_model_attention_by_hand():
    # two tokens, scores ln 1 and ln 3: weights 1/4 and 3/4
    q = np.array([[[np.log(3.0)] + [0.0] * 63]])
    k = np.zeros((2, 1, 64))
    k[1, 0, 0] = 1.0
    v = np.stack([np.full((1, 64), 4.0), np.full((1, 64), 8.0)])
    out, lse, _, _ = ref.attend(q, k, v, None, np.ones(2, bool), [1], None, 1.0, True, 0, 0, 0.0, None)
    assert np.allclose(out, 7.0) and np.allclose(lse, np.log(4.0))
    out, lse, _, _ = ref.attend(q, k, v, None, np.ones(2, bool), [0], None, 1.0, True, 0, 0, 0.0, None)
    assert np.allclose(out, 4.0) and np.allclose(lse, 0.0)
    out, lse, _, _ = ref.attend(q, k, v, None, np.ones(2, bool), [-1], None, 1.0, True, 0, 0, 0.0, None)
    assert np.all(out == 0) and np.isneginf(lse).all()
