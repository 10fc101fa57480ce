"""The latent calls as they are used together: a conversation appended and attended
step by step, streams, graphs, large pools, the example."""
import importlib.util
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import kv_reference as kv
import latent_reference as ref
import paper_2607_05708_amd as pm
from test_gpu_kv_streams import allocations
from test_gpu_latent import FORMS, Problem, host, up

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("fmt", [pm.MEM_KV_BF16, pm.MEM_KV_FP8, pm.MEM_KV_FP4])
def test_a_conversation_step_by_step(fmt):
    # a prompt, drafted tokens, then single ones: appended with their rotation, attended at once, each step against the
    # model over what the cache holds by then
    h, d, latent, T, ppc = 4, 64, 256, 32, 2
    rng = np.random.default_rng(fmt)
    f = (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    pool = np.full((12, ref.page_bytes(fmt, T, latent) + 48), 255, np.uint8)  # (pages longer than they need to be)
    table = rng.permutation(12).reshape(6, ppc).astype(np.int32)
    cache = pm.LatentCache(up(pool), up(table), T, latent, ref.ROPE, fmt)
    w = (torch.randn((h, 2 * d, latent), device="cuda") / 16).to(torch.bfloat16)
    w64 = host(w)
    order = np.array([4, 1, 3], np.int32)                    # the conversation's chunks
    held, context = 0, []
    for n in (70, 5, 1, 1, 40, 1):
        x = torch.randn((n, latent + ref.ROPE), device="cuda").to(torch.bfloat16)
        q = torch.randn((n, h, d + ref.ROPE), device="cuda").to(torch.bfloat16)
        at = held + np.arange(n)
        chunk, pos = order[at // (T * ppc)], at % (T * ppc)
        t = pm.mem_latent_append(cache, x[:, :latent], x[:, latent:], up(chunk.astype(np.int32)),
                                 up(pos.astype(np.int32)), up(at.astype(np.int32)), up(f), q=q[..., d:])
        held += n
        tok_len = np.zeros(6, np.int32)
        tok_len[order] = np.clip(held - np.arange(3) * T * ppc, 0, T * ppc)
        context += [(table[c, p // T], p % T) for c, p in zip(chunk, pos)]
        host_pool = cache.pool.cpu().numpy()
        page, row = (np.array([c[j] for c in context]) for j in (0, 1))
        c, r = ref.get(fmt, T, latent, host_pool, page, row)
        want_t = kv.to_bf16(ref.rotate(host(q[..., d:]), at, f, False))
        assert np.array_equal(host(t), want_t)
        for form in FORMS:
            lse = torch.empty((n, h), device="cuda")
            out = pm.mem_latent_attend(cache, up(tok_len), up(order[None]), q[..., :d], t, w, 0.09, causal=True,
                                       form=form, lse=lse)
            model = ref.attend(form, host(q[..., :d]), want_t, c, r, w64, None, np.ones(held, bool), at, None,
                               float(np.float32(0.09)), True, 0, 0)
            ref.check_attend(f"{n} tokens, form {form}", host(out), host(lse), *model)


def test_rotated_keys_attended():
    # scores of rotated keys and queries depend on distances alone: the whole context moved by 1,000 positions
    n, h, d, T = 60, 2, 64, 32
    f = up((10000.0 ** (-np.arange(32) / 32)).astype(np.float32))
    k, v, q = (torch.randn((n, x, d), device="cuda").to(torch.bfloat16) for x in (1, 1, h))
    chunk, pos = up(np.zeros(n, np.int32)), up(np.arange(n, dtype=np.int32))
    outs = []
    for shift in (0, 1000):
        pool = torch.zeros((2, kv.page_bytes(kv.BF16, T, 1, d)), dtype=torch.uint8, device="cuda")
        cache = pm.KvCache(pool, up(np.arange(2, dtype=np.int32)[None]), T, 1, d, pm.MEM_KV_BF16)
        turned = pm.mem_kv_append(cache, k, v, chunk, pos, pos + shift, f, q=q)
        outs.append(host(pm.mem_attend(cache, up(np.array([n], np.int32)), up(np.zeros((1, 1), np.int32)), turned,
                                       0.125, causal=True)[0]))
    # keys and queries are rounded to bf16 after their rotation, 2^-9 of each on average: a score of some 64 products of
    # that size moves by less than 0.125 * 6 * 2^-8 * sqrt(2 * 64) * 4 = 1 / 8 once in 3e7, a weight by e^(1/4)
    assert np.abs(outs[0] - outs[1]).max() < 4 * (np.exp(0.25) - 1)
    assert np.abs(outs[0] - outs[1]).mean() < 0.02


def test_calls_on_another_stream_take_that_streams_memory(monkeypatch):
    p = Problem(31, pm.MEM_KV_FP8, [[64] * 12, [64, 5]], [3, 3], 4, 64, 256)
    cache, q, t, w = p.cache(), p.q.cuda(), p.t.cuda(), p.w.cuda()
    off, tok, ids = up(p.off), up(p.tok_len), up(p.ids)
    chunk, pos = up(np.full(20, -1, np.int32)), up(np.arange(20, dtype=np.int32))
    x, rows = torch.randn((20, 320), device="cuda"), torch.randn((20, 3, 64), device="cuda")
    f = up(np.ones(32, np.float32))
    calls = [(2, lambda s: pm.mem_latent_read(cache, chunk, pos, stream=s)),
             (1, lambda s: [pm.mem_latent_append(cache, x[:, :256], x[:, 256:], chunk, pos, pos, f, q=rows, stream=s)]),
             *[(2, lambda s, form=form: [pm.mem_latent_attend(cache, tok, ids, q, t, w, p.scale, q_offsets=off,
                                                              causal=True, form=form, stream=s)]) for form in FORMS]]
    side = torch.cuda.Stream()
    for count, call in calls:
        want, here = allocations(monkeypatch, lambda: call(None))
        assert [s for s, _, _ in here] == [torch.cuda.current_stream().cuda_stream] * count
        want = [a.clone() for a in want]
        torch.cuda.synchronize()
        got, there = allocations(monkeypatch, lambda: call(side))
        assert [s for s, _, _ in there] == [side.cuda_stream] * count
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_offsets_beyond_32_bits():
    # pages behind the first 4 GiB of the pool
    fmt, T, latent, h, d = pm.MEM_KV_BF16, 64, 512, 3, 128
    page = ref.page_bytes(fmt, T, latent)
    n_pages = (5 << 30) // page
    pool = torch.zeros((n_pages, page), dtype=torch.uint8, device="cuda")
    table = np.array([[n_pages - 1, n_pages - 3], [n_pages - 2, 1]], np.int32)
    cache = pm.LatentCache(pool, up(table), T, latent, ref.ROPE, fmt)
    n = 200
    at = np.arange(n)
    chunk, pos = (at // 128).astype(np.int32), (at % 128).astype(np.int32)
    x = torch.randn((n, latent + ref.ROPE), device="cuda").to(torch.bfloat16)
    pm.mem_latent_append(cache, x[:, :latent], x[:, latent:], up(chunk), up(pos))
    c, r = pm.mem_latent_read(cache, up(chunk), up(pos))
    assert torch.equal(c, x[:, :latent]) and torch.equal(r, x[:, latent:])
    q = torch.randn((n, h, d + ref.ROPE), device="cuda").to(torch.bfloat16)
    w = (torch.randn((h, 2 * d, latent), device="cuda") / 22).to(torch.bfloat16)
    model = {}
    for form in FORMS:
        lse = torch.empty((n, h), device="cuda")
        out = pm.mem_latent_attend(cache, up(np.array([128, 72], np.int32)), up(np.array([[0, 1]], np.int32)),
                                   q[..., :d], q[..., d:], w, 0.07, causal=True, form=form, lse=lse)
        model[form] = ref.attend(form, host(q[..., :d]), host(q[..., d:]), host(c), host(r), host(w), None,
                                 np.ones(n, bool), at, None, float(np.float32(0.07)), True, 0, 0)
        ref.check_attend(f"form {form}", host(out), host(lse), *model[form])


@pytest.mark.parametrize("form", FORMS)
def test_rows_that_see_nothing_are_zero_whatever_the_weights_hold(form):
    p = Problem(3, pm.MEM_KV_FP8, [[], [64, 10]], [2, 3], 2, 64, 256)
    w = p.w.cuda()
    w[:, 70], w[:, 80] = float("inf"), float("nan")
    out, lse = p.gpu(form, w=w)
    assert (out[:2] == 0).all() and np.isneginf(lse[:2]).all()
    assert not np.isfinite(out[2:, :, 6]).any() and not np.isfinite(out[2:, :, 16]).any()
    if form == pm.MEM_LATENT_ABSORBED:                      # (in the expanded form they make a token's values so)
        assert np.isfinite(out[2:, :, 7:16]).all()


@pytest.mark.parametrize("form", FORMS)
def test_pages_stay_a_cache_when_they_are_moved(form):
    p = Problem(9, pm.MEM_KV_FP4, [[64, 64, 30]], [4], 3, 64, 256)
    want = p.gpu(form)
    ids = up(p.ids[0])
    moved = pm.mem_gather_chunks(up(p.pool), up(p.table), ids, pm.MEM_ORDER_RANK, 1)
    ppc = p.table.shape[1]
    cache = pm.LatentCache(moved.view(-1, p.pool.shape[1]), up(np.arange(3 * ppc, dtype=np.int32).reshape(3, ppc)), 32,
                           256, ref.ROPE, p.fmt)
    p.tok_len, p.ids = p.tok_len[p.ids[0]], np.arange(3, dtype=np.int32)[None]
    got = p.gpu(form, cache=cache)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_a_turn_as_a_graph():
    # append and both forms of attention captured as one graph, replayed with other inputs and eager work in between
    n, h, d, latent, T = 40, 2, 64, 256, 32
    pool = torch.zeros((2, ref.page_bytes(pm.MEM_KV_FP8, T, latent)), dtype=torch.uint8, device="cuda")
    cache = pm.LatentCache(pool, up(np.arange(2, dtype=np.int32)[None]), T, latent, ref.ROPE, pm.MEM_KV_FP8)
    x = torch.empty((n, latent + ref.ROPE), device="cuda", dtype=torch.bfloat16)
    q = torch.empty((n, h, d + ref.ROPE), device="cuda", dtype=torch.bfloat16)
    w = (torch.randn((h, 2 * d, latent), device="cuda") / 16).to(torch.bfloat16)
    chunk, pos = up(np.zeros(n, np.int32)), up(np.arange(n, dtype=np.int32))
    f, tok, ids = up(np.linspace(1, 0, 32).astype(np.float32)), up(np.array([n], np.int32)), up(np.zeros((1, 1), np.int32))

    def turn():
        t = pm.mem_latent_append(cache, x[:, :latent], x[:, latent:], chunk, pos, pos, f, q=q[..., d:])
        return [t] + [pm.mem_latent_attend(cache, tok, ids, q[..., :d], t, w, 0.1, causal=True, form=form)
                      for form in FORMS]

    def fresh(seed):
        g = torch.Generator("cuda").manual_seed(seed)
        for a in (x, q):
            a.copy_(torch.randn(a.shape, device="cuda", generator=g))

    fresh(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        turn()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = turn()
    for seed in (1, 2, 3):
        fresh(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [a.clone() for a in kept]
        assert all(torch.equal(a, b) for a, b in zip(got, turn()))


def test_example():
    path = os.path.join(ROOT, "examples", "latent_memory.py")
    r = subprocess.run([sys.executable, path], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr
    assert len(r.stdout.strip().splitlines()) == 3
    spec = importlib.util.spec_from_file_location("latent_memory", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    g = torch.Generator("cuda").manual_seed(5)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    mem = ex.Memory(64)
    past = mem.open(rand(8, ex.EMB))
    mem.store(past, rand(8 * 33, ex.LATENT + ex.ROPE), past * 512)
    w = (rand(ex.HEADS, 2 * ex.HEAD_DIM, ex.LATENT).float() / 22).to(torch.bfloat16)
    q, x = rand(2, ex.HEADS, ex.HEAD_DIM + ex.ROPE), rand(2, ex.LATENT + ex.ROPE)
    start = torch.tensor([5000, 6000], dtype=torch.int32, device="cuda")
    out, ids = ex.turn(mem, rand(2, ex.EMB), q, x, w, start, top=3)
    pool, table, ids = mem.cache.pool.cpu().numpy(), mem.cache.table.cpu().numpy(), ids.cpu().numpy()
    freq = mem.freq.cpu().numpy()
    for i in range(2):
        lens = [33, 33, 33, 1]
        where = [(table[c, j // 64], j % 64) for c, m in zip(ids[i], lens) for j in range(m)]
        c, r = ref.get(pm.MEM_KV_FP8, 64, ex.LATENT, pool, *(np.array([v[j] for v in where]) for j in (0, 1)))
        t = kv.to_bf16(ref.rotate(host(q[i:i + 1, :, ex.HEAD_DIM:]), [int(start[i])], freq, True))
        model = ref.attend(ref.ABSORBED, host(q[i:i + 1, :, :ex.HEAD_DIM]), t, c, r, host(w), None, np.ones(100, bool),
                           [99], None, float(np.float32(1 / np.sqrt(192))), True, 0, 0)
        ref.check_attend("turn", host(out[i:i + 1]), model[1], *model)
