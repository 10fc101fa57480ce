"""Seeded sweeps of the latent calls over sizes, masks and layouts together, and documented calls at the edges: caches
without a page, offsets that leave all rows to nobody, weights that heads share, rows of no stride."""
import numpy as np
import pytest
import torch

import kv_reference as kv
import latent_reference as ref
import paper_2607_05708_amd as pm
from test_gpu_latent import FMTS, FORMS, Problem, host, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("seed", range(40))
def test_sweep(seed):
    rng = np.random.default_rng(1000 + seed)
    name = rng.choice(list(FMTS))
    latent, d = rng.choice([256, 512]), rng.choice([64, 128])
    T, ppc = rng.choice([32, 64, 96]), rng.integers(1, 5)
    h, m = int(rng.choice([1, 2, 5, 8, 17, 33])), int(rng.integers(1, 7))
    room = T * ppc
    lens = [[int(x) for x in rng.integers(0, room + 1, rng.integers(0, 6))] for _ in range(m)]
    nq = [int(x) for x in rng.choice([0, 1, 2, 3, 7, 19, 40], m)]
    nq[rng.integers(m)] += 1
    docs = int(rng.choice([0, 0, 3]))
    k = max(1, max(len(x) for x in lens)) + int(rng.integers(0, 5))
    p = Problem(seed, FMTS[name], lens, nq, h, int(d), int(latent), page_tokens=int(T), ppc=int(ppc), k=k, docs=docs,
                holes=bool(rng.random() < 0.5), spread=float(rng.choice([0.1, 1.0, 4.0])))
    total = len(p.q)
    masks = dict(causal=bool(rng.random() < 0.6), window=int(rng.choice([0, 0, 1, 33, 200])))
    if rng.random() < 0.4:
        masks["prefix"] = rng.integers(-5, room, m)
    if rng.random() < 0.4:
        masks["q_pos"] = rng.integers(-3, 5 * room, total)
    p.check(f"seed {seed}: {name} {latent} {d}, {h} heads, {nq} over {lens}, {masks}", **masks)


@pytest.mark.parametrize("form", FORMS)
def test_a_cache_without_pages(form):
    fmt, h, d, latent = pm.MEM_KV_FP8, 3, 64, 256
    cache = pm.LatentCache(torch.empty((0, ref.page_bytes(fmt, 32, latent)), dtype=torch.uint8, device="cuda"),
                           up(np.array([[0, 5], [-1, 2 ** 31 - 1]], np.int32)), 32, latent, ref.ROPE, fmt)
    x = torch.randn((4, h, d + ref.ROPE), device="cuda").to(torch.bfloat16)
    w = torch.randn((h, 2 * d, latent), device="cuda").to(torch.bfloat16)
    lse = torch.full((4, h), 7.0, device="cuda")
    out = pm.mem_latent_attend(cache, up(np.array([64, 9], np.int32)), up(np.array([[0, 1], [1, 0]], np.int32)),
                               x[..., :d], x[..., d:], w, 0.1, form=form, lse=lse)
    assert (host(out) == 0).all() and np.isneginf(host(lse)).all()
    none = pm.LatentCache(cache.pool, torch.empty((0, 2), dtype=torch.int32, device="cuda"), 32, latent, ref.ROPE, fmt)
    out = pm.mem_latent_attend(none, up(np.zeros(0, np.int32)), up(np.array([[0, -1], [3, 0]], np.int32)), x[..., :d],
                               x[..., d:], w, 0.1, form=form, lse=lse.fill_(7.0))
    assert (host(out) == 0).all() and np.isneginf(host(lse)).all()
    some = up(np.array([0, 1, 1], np.int32))
    ones = up(np.ones(32, np.float32))
    with pytest.raises(ValueError):                         # elements of no stride
        pm.mem_latent_append(none, x[:3, 0, :1].expand(3, latent), x[:3, 0, d:], some, some)
    t = pm.mem_latent_append(none, x[:1].view(1, -1)[:, :latent].expand(3, latent), x[:3, 0, d:], some, some, some, ones,
                             q=x[:3, :, d:])
    want = kv.to_bf16(ref.rotate(host(x[:3, :, d:]), [0, 1, 1], np.ones(32), False))
    assert np.array_equal(host(t), want)
    c, r = pm.mem_latent_read(none, some, some)
    assert not host(c).any() and not host(r).any()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("m", [3, 600])
def test_offsets_that_leave_all_rows_to_nobody(form, m):
    p = Problem(4, FMTS["fp4"], [[64, 10]] + [[]] * (m - 1), [5] + [0] * (m - 1), 4, 64, 256)
    for at in (0, 5):
        out = torch.full((5, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16)
        lse = torch.full((5, 4), 7.0, device="cuda")
        pm.mem_latent_attend(p.cache(), up(p.tok_len), up(p.ids), p.q.cuda(), p.t.cuda(), p.w.cuda(), p.scale,
                             q_offsets=up(np.full(m + 1, at, np.int32)), form=form, out=out, lse=lse)
        assert (host(out) == 7).all() and (host(lse) == 7).all()


@pytest.mark.parametrize("form", FORMS)
def test_weights_and_rows_without_a_stride(form):
    # all heads with the same weights, all tokens with the same query
    p = Problem(6, FMTS["bf16"], [[64, 40]], [3], 5, 64, 256)
    p.w, p.q = p.w[:1].repeat(5, 1, 1), p.q[:1].repeat(3, 1, 1)
    want = p.gpu(form)
    got = p.gpu(form, w=p.w[:1].cuda().expand(5, 128, 256), q=p.q[:1].cuda().expand(3, 5, 64))
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    ref.check_attend("shared", *want, *p.model(form))


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("n", [1, 5, 700])
def test_queries_rotated_in_place_in_a_fused_array(pairs, n):
    # [q heads | latent vector | key part] of a token in one array: q is rotated where it lies, the rest stays
    h, latent, fmt = 3, 256, pm.MEM_KV_BF16
    rng = np.random.default_rng(n)
    width = h * 64 + latent + 64
    x = torch.from_numpy(rng.standard_normal((n, width)).astype(np.float32)).to(torch.bfloat16)
    g = x.cuda()
    pages = -(-n // 32)
    cache = pm.LatentCache(torch.zeros((pages, ref.page_bytes(fmt, 32, latent)), dtype=torch.uint8, device="cuda"),
                           up(np.arange(pages, dtype=np.int32)[:, None]), 32, latent, ref.ROPE, fmt)
    at, f = rng.integers(-2 ** 31, 2 ** 31, n), (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    i = np.arange(n)
    q = g[:, :h * 64].view(n, h, 64)
    back = pm.mem_latent_append(cache, g[:, h * 64:h * 64 + latent], g[:, h * 64 + latent:], up((i // 32).astype(np.int32)),
                                up((i % 32).astype(np.int32)), up(at.astype(np.int32)), up(f), q=q, q_out=q, pairs=pairs)
    assert back is q
    x = x.double().numpy()
    assert np.array_equal(host(q), kv.to_bf16(ref.rotate(x[:, :h * 64].reshape(n, h, 64), at, f, pairs)))
    assert np.array_equal(host(g[:, h * 64:]), x[:, h * 64:])
    c, r = pm.mem_latent_read(cache, up((i // 32).astype(np.int32)), up((i % 32).astype(np.int32)))
    assert np.array_equal(host(c), x[:, h * 64:h * 64 + latent])
    assert np.array_equal(host(r), kv.to_bf16(ref.rotate(x[:, None, h * 64 + latent:], at, f, pairs))[:, 0])
