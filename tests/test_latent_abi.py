"""The append and latent calls without a GPU: declarations, sizes, refusals before
any launch, the binding's own checks, and the 64-bit model's pins."""
import ctypes as C
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2607_05708_amd as pm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INCLUDE = os.path.join(ROOT, "include")
FAKE = 0x100000  # never dereferenced: every call below fails validation first

needs_lib = pytest.mark.skipif(not os.path.exists(pm.library_path()), reason="libmemattn.so not built")


def declared(header):
    text = open(os.path.join(INCLUDE, header)).read()
    return sorted(set(re.findall(r"MEMATTN_API\s+[\w\s\*]+?\b(mem_\w+)\s*\(", text)))


def test_headers_declare_the_calls():
    assert declared("memattn_append.h") == ["mem_kv_append"]
    assert declared("memattn_latent.h") == ["mem_latent_append", "mem_latent_attend",
                                            "mem_latent_attend_workspace_bytes", "mem_latent_page_bytes",
                                            "mem_latent_read"]


@needs_lib
def test_library_exports_every_declared_symbol():
    L = C.CDLL(pm.library_path())
    for name in declared("memattn_append.h") + declared("memattn_latent.h"):
        assert hasattr(L, name), name


@pytest.mark.skipif(shutil.which("gcc") is None or shutil.which("g++") is None, reason="gcc/g++ not available")
@pytest.mark.parametrize("header", ["memattn_append.h", "memattn_latent.h"])
def test_header_is_c99_and_cxx17(header):
    for cmd in (["gcc", "-std=c99", "-pedantic", "-x", "c"], ["g++", "-std=c++17", "-x", "c++"]):
        r = subprocess.run([*cmd, "-Wall", "-Wextra", "-Werror", "-fsyntax-only", os.path.join(INCLUDE, header)],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr


@needs_lib
def test_page_bytes():
    for fmt, t, l in ((0, 64, 512), (1, 32, 256), (2, 256, 512), (2, 32, 256)):
        assert pm.mem_latent_page_bytes(t, l, 64, fmt) == ref.page_bytes(fmt, t, l)
        assert pm.mem_latent_page_bytes(t, l, 64, fmt) % 16 == 0
    for bad in ((64, 512, 64, 3), (64, 512, 64, -1), (64, 384, 64, 2), (48, 512, 64, 2), (0, 512, 64, 2),
                (8192, 512, 64, 2), (64, 512, 32, 2), (64, 0, 64, 2)):
        assert pm.mem_latent_page_bytes(*bad) == 0
    for i in range(4):
        sizes = [64, 512, 64, 2]
        sizes[i] = 2 ** 32 + sizes[i]
        with pytest.raises(ValueError):
            pm.mem_latent_page_bytes(*sizes)


def _kv(**kw):
    a = dict(pool=FAKE, n_pages=64, page_bytes=69632, table=FAKE, n_chunks=8, ppc=8, page_tokens=64, heads=8,
             head_dim=128, format=pm.MEM_KV_FP4)
    a.update(kw)
    return pm.MemKv(pm.MemPages(a["pool"], a["n_pages"], a["page_bytes"], a["table"], a["n_chunks"], a["ppc"]),
                    a["page_tokens"], a["heads"], a["head_dim"], a["format"])


def _latent(**kw):
    a = dict(pool=FAKE, n_pages=64, page_bytes=64 * 400, table=FAKE, n_chunks=8, ppc=8, page_tokens=64, latent_dim=512,
             rope_dim=64, format=pm.MEM_KV_FP4)
    a.update(kw)
    return pm.MemLatent(pm.MemPages(a["pool"], a["n_pages"], a["page_bytes"], a["table"], a["n_chunks"], a["ppc"]),
                        a["page_tokens"], a["latent_dim"], a["rope_dim"], a["format"])


BAD_PAGES = [(dict(format=3), -1), (dict(format=-1), -1), (dict(page_tokens=48), -1), (dict(page_tokens=0), -1),
             (dict(page_tokens=4128), -1), (dict(ppc=0), -1), (dict(ppc=65), -1), (dict(n_pages=-1), -1),
             (dict(n_chunks=-1), -1), (dict(n_pages=1 << 31), -2), (dict(n_chunks=1 << 31), -2),
             (dict(page_bytes=0), -1), (dict(page_bytes=64 * 400 - 16), -1), (dict(page_bytes=64 * 400 + 8), -1),
             (dict(pool=None), -1), (dict(table=None), -1), (dict(pool=FAKE + 8), -1), (dict(table=FAKE + 2), -1)]
BAD_LATENT = BAD_PAGES + [(dict(latent_dim=0), -1), (dict(latent_dim=384), -2), (dict(latent_dim=1024), -2),
                          (dict(rope_dim=0), -1), (dict(rope_dim=32), -2)]
FAR = 0x10000000


def _rows(data=FAR, ts=8192, hs=128):
    return pm.MemKvRows(data, ts, hs)


def _rot(pos=FAKE, freq=FAKE, dim=64, style=0):
    return pm.MemRotation(pos, freq, dim, style)


def _p(x):
    return None if x is None else C.byref(x)


def _common_append_refusals(go):
    """What both appends refuse; go(**kw) calls one of them with some arguments changed."""
    assert go(a=None) == -1 and go(b=None) == -1
    assert go(a=_rows(None)) == -1 and go(b=_rows(FAR + 1)) == -1 and go(a=_rows(ts=-1)) == -1
    assert go(dtype=2) == -1 and go(n=-1) == -1 and go(chunk=None) == -1 and go(pos=FAKE + 1) == -1
    assert go(n=1 << 40) == -2
    assert go(rot=_rot(pos=None)) == -1 and go(rot=_rot(freq=None)) == -1 and go(rot=_rot(freq=FAKE + 2)) == -1
    assert go(rot=_rot(style=2)) == -1 and go(rot=_rot(dim=24)) == -1 and go(rot=_rot(dim=0)) == -1
    assert go(n=0) == 0
    q, o = _rows(2 * FAR), _rows(3 * FAR)
    for kw in (dict(q=q, heads_q=4), dict(q_out=o, heads_q=4), dict(q=q, q_out=o), dict(heads_q=4),
               dict(q=q, q_out=o, heads_q=-1), dict(q=q, q_out=o, heads_q=1025)):
        assert go(**kw) == -1, kw
    assert go(q=q, q_out=_rows(3 * FAR, hs=32), heads_q=4) == -1            # rows of q_out overlap
    assert go(q=q, q_out=_rows(FAKE + 4096), heads_q=4) == -1               # the pool
    assert go(q=q, q_out=_rows(2 * FAR + 64), heads_q=4) == -1              # q, but not the same rows
    assert go(q=q, q_out=_rows(2 * FAR), heads_q=4, dtype=pm.MEM_F32) == -1  # in place, but of other elements
    assert go(q=q, q_out=_rows(FAR), heads_q=4) == -1                       # the first rows
    assert b"apart" in pm.lib().mem_last_error()


@needs_lib
def test_kv_append_refusals():
    def go(kv=_kv(), a=_rows(), b=_rows(FAR + 4096), q=None, q_out=None, heads_q=0, dtype=pm.MEM_BF16, rot=_rot(),
           chunk=FAKE, pos=FAKE, n=4):
        return pm.lib().mem_kv_append(_p(kv), _p(a), _p(b), _p(q), _p(q_out), heads_q, dtype, _p(rot), chunk, pos, n,
                                      None)

    for kw, status in BAD_PAGES[:11] + [(dict(heads=0), -1), (dict(head_dim=96), -2), (dict(page_bytes=0), -1),
                                        (dict(page_bytes=69616), -1), (dict(pool=None), -1), (dict(table=None), -1)]:
        assert go(kv=_kv(**kw)) == status, kw
        assert pm.lib().mem_last_error()
    assert go(kv=None) == -1 and go(rot=None) == -1
    assert go(rot=_rot(dim=144)) == -1
    _common_append_refusals(go)


@needs_lib
def test_latent_append_refusals():
    def go(cache=_latent(), a=_rows(), b=_rows(FAR + 4096), q=None, q_out=None, heads_q=0, dtype=pm.MEM_BF16,
           rot=_rot(), chunk=FAKE, pos=FAKE, n=4):
        return pm.lib().mem_latent_append(_p(cache), _p(a), _p(b), _p(q), _p(q_out), heads_q, dtype, _p(rot), chunk,
                                          pos, n, None)

    for kw, status in BAD_LATENT:
        assert go(cache=_latent(**kw)) == status, kw
        assert pm.lib().mem_last_error()
    assert go(cache=None) == -1
    assert go(rot=_rot(dim=32)) == -1
    assert go(rot=None, q=_rows(2 * FAR), q_out=_rows(3 * FAR), heads_q=2) == -1
    _common_append_refusals(go)


@needs_lib
def test_latent_read_refusals():
    def go(cache=_latent(), c=_rows(), r=_rows(2 * FAR), dtype=pm.MEM_BF16, chunk=FAKE, pos=FAKE, n=4):
        return pm.lib().mem_latent_read(_p(cache), _p(c), _p(r), dtype, chunk, pos, n, None)

    for kw, status in BAD_LATENT:
        assert go(cache=_latent(**kw)) == status, kw
    assert go(cache=None) == -1 and go(c=None) == -1 and go(r=_rows(None)) == -1
    assert go(c=_rows(FAR + 1)) == -1 and go(r=_rows(ts=-1)) == -1
    assert go(dtype=5) == -1 and go(chunk=None) == -1 and go(pos=None) == -1 and go(chunk=FAKE + 1) == -1
    assert go(n=-1) == -1 and go(n=1 << 40) == -2 and go(n=0) == 0
    assert go(c=_rows(ts=511)) == -1 and go(r=_rows(2 * FAR, ts=32)) == -1 and go(c=_rows(ts=0)) == -1
    assert go(c=_rows(FAKE + 4096)) == -1 and go(r=_rows(FAKE + 4096)) == -1
    assert go(r=_rows(FAR + 2 * 256)) == -1                                  # between the elements of c
    assert b"apart" in pm.lib().mem_last_error()


@needs_lib
def test_latent_attend_refusals():
    L = pm.lib()

    def go(cache=_latent(), q=_rows(), t=_rows(2 * FAR), total_q=4, w=True, form=0, out=FAKE, lse=FAKE, ws=FAKE,
           ws_bytes=1 << 40, args=True, **kw):
        a = dict(tok_len=FAKE, ids=FAKE, m=4, k=8, heads_q=32, q_offsets=None, q_pos=None, scale=0.1, softcap=0.0,
                 slopes=None, causal=0, window=0, prefix_len=None, chunk_ns=None, query_ns=None)
        wt = dict(data=FAKE, head_stride=256 * 512, row_stride=512, head_dim=128)
        for x in list(kw):
            (wt if x in wt else a)[x] = kw.pop(x)
        arg, weights = pm.MemAttendArgs(*a.values()), pm.MemLatentWeights(*wt.values())
        return L.mem_latent_attend(_p(cache), C.byref(arg) if args else None, _p(q), _p(t), total_q,
                                   C.byref(weights) if w else None, form, out, lse, ws, ws_bytes, None)

    for kw, status in BAD_LATENT:
        assert go(cache=_latent(**kw)) == status, kw
    inf, nan = float("inf"), float("nan")
    for kw in (dict(cache=None), dict(args=False), dict(w=False), dict(m=-1), dict(total_q=-1), dict(k=0), dict(k=4097),
               dict(heads_q=0), dict(heads_q=1025), dict(scale=0.0), dict(scale=nan), dict(scale=inf), dict(scale=-1.0),
               dict(softcap=-1.0), dict(softcap=nan), dict(window=-1), dict(m=0), dict(m=3), dict(ids=None),
               dict(tok_len=None), dict(chunk_ns=FAKE), dict(q=None), dict(t=None), dict(q=_rows(FAR + 1)),
               dict(t=_rows(ts=-1)), dict(out=None), dict(out=FAKE + 8), dict(ids=FAKE + 2), dict(lse=FAKE + 2),
               dict(data=None), dict(data=FAKE + 8), dict(head_stride=-8), dict(row_stride=4), dict(head_dim=0),
               dict(form=3), dict(form=-1), dict(ws=FAKE + 8)):
        assert go(**kw) == -1, kw
        assert L.mem_last_error()
    for kw in (dict(head_dim=96), dict(head_dim=256), dict(softcap=30.0), dict(slopes=FAKE)):
        assert go(**kw) == -2, kw
    for form in (1, 2):
        need = L.mem_latent_attend_workspace_bytes(C.byref(_latent()), 4, 8, 4, 32, 128, form)
        assert need > 0 and need % 16 == 0
        assert go(form=form, ws=None) == -3 and go(form=form, ws_bytes=need - 1) == -3
        # what is written, on itself or on what is read: q and w at FAR and FAKE, the pool and the workspace further on
        far = dict(q=_rows(), t=_rows(2 * FAR), data=3 * FAR, out=4 * FAR, lse=5 * FAR, ws=6 * FAR, form=form)
        for kw, names in ((dict(out=FAR), b"out overlaps q"), (dict(out=2 * FAR), b"out overlaps t"),
                          (dict(out=3 * FAR), b"out overlaps w"), (dict(lse=FAR), b"lse overlaps q"),
                          (dict(lse=4 * FAR), b"out overlaps lse"), (dict(ws=4 * FAR - 16), b"out overlaps workspace"),
                          (dict(ws=2 * FAR), b"workspace overlaps t"), (dict(out=FAKE), b"out overlaps the page pool")):
            assert go(**{**far, **kw}) == -1 and L.mem_last_error() == names, (kw, L.mem_last_error())
    for kw in (dict(head_stride=1 << 45), dict(row_stride=1 << 45)):
        assert go(**kw) == -1 and b"out of memory" in L.mem_last_error()
    assert go(total_q=1 << 26, m=1 << 26) == -2 and go(total_q=(1 << 30) // 32 + 1, m=1) == -2
    assert go(total_q=0) == 0 and go(total_q=0, m=0) == 0
    for total, m, heads, form in ((1 << 24, 1 << 24, 1, 2), (1 << 30, 1, 1, 1), (1 << 24, 1 << 24, 1, 1)):
        assert go(total_q=total, m=m, heads_q=heads, form=form, ws_bytes=1 << 62) == -2   # more than one launch


@needs_lib
def test_workspace_sizes():
    size = lambda c, *a: pm.lib().mem_latent_attend_workspace_bytes(C.byref(c), *a)  # noqa: E731
    for bad in ((_latent(format=9), 4, 8, 4, 32, 128, 0), (_latent(), -1, 8, 4, 32, 128, 0),
                (_latent(), 4, 0, 4, 32, 128, 0), (_latent(), 4, 8, -1, 32, 128, 0), (_latent(), 4, 8, 4, 0, 128, 0),
                (_latent(), 4, 8, 4, 32, 96, 0), (_latent(), 4, 8, 4, 32, 128, 7), (_latent(), 0, 8, 0, 32, 128, 0)):
        assert size(*bad) == 0
    # the form that is chosen: few new tokens a request absorbed, many expanded
    few, many = (_latent(), 4, 8, 4, 32, 128), (_latent(), 4, 8, 8192, 32, 128)
    assert size(*few, 0) == size(*few, 1) != size(*few, 2) and size(*many, 0) == size(*many, 2) != size(*many, 1)
    # keys and values of a call's context are made a part of the heads at a time: some 1 GiB at most, or one head
    chunk = 4096 * 64 * 4096 // 2                               # tokens that the longest list can hold, half of them
    assert size(_latent(ppc=1), 64, 64, 64 * 2048, 128, 128, 2) < 3 << 29
    assert size(_latent(page_tokens=4096, ppc=64, page_bytes=4096 * 400), 1, 2048, 2048, 128, 128, 2) < chunk * 800


def test_bindings_refuse_host_tensors():
    cpu = torch.zeros((4, 64 * 400), dtype=torch.uint8)
    with pytest.raises(ValueError):
        pm.LatentCache(cpu, torch.zeros((1, 4), dtype=torch.int32), 64, 512, 64, pm.MEM_KV_FP4)


# ---------------------------------------------------------------- the model itself

def test_model_rotation_by_hand():
    x = np.zeros((3, 2, 6))
    x[..., 0], x[..., 2], x[..., 4] = 1.0, 2.0, 5.0
    f = np.array([np.pi / 2, np.pi], np.float64)
    y = ref.rotate(x, [0, 1, 2], f, False)                      # pairs (0, 2), (1, 3); 4 and 5 stay
    assert np.allclose(y[0], x[0])
    assert np.allclose(y[1, :, 0], -2) and np.allclose(y[1, :, 2], 1) and np.allclose(y[1, :, 4], 5)
    assert np.allclose(y[2, :, 0], -1) and np.allclose(y[2, :, 2], -2)
    y = ref.rotate(x, [0, 1, 2], f, True)                       # pairs (0, 1), (2, 3)
    assert np.allclose(y[1, :, 1], 1) and np.allclose(y[1, :, 0], 0) and np.allclose(y[1, :, 2], -2)
    # what a rotated key's product with a rotated query depends on is their distance
    rng = np.random.default_rng(0)
    q, k, f = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64)), rng.random(32)
    a, b = ((ref.rotate(q, [p + 7], f, s) * ref.rotate(k, [p], f, s)).sum() for p, s in ((0, True), (100, True)))
    assert np.isclose(a, b)


def test_model_forms_agree():
    rng = np.random.default_rng(1)
    q, t, w = rng.standard_normal((2, 3, 64)), rng.standard_normal((2, 3, 64)), rng.standard_normal((3, 128, 256)) / 16
    c, r = rng.standard_normal((9, 256)), rng.standard_normal((9, 64))
    args = (q, t, c, r, w, None, np.ones(9, bool), [3, 8], None, 0.1, True, 0, 0)
    a, b = ref.attend(ref.ABSORBED, *args), ref.attend(ref.EXPANDED, *args)
    assert np.abs(a[0] - b[0]).max() < 0.02 and np.abs(a[1] - b[1]).max() < 0.02
    p = np.exp(0.1 * ((q[0, 1] @ w[1, :64]) @ c[:4].T + t[0, 1] @ r[:4].T))
    assert np.allclose(a[0][0, 1], (p @ c[:4]) @ w[1, 64:].T / p.sum(), atol=0.02)
