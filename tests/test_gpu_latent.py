"""Latent attention on the GPU, both forms, against the 64-bit model of
latent_reference.py."""
import itertools

import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2607_05708_amd as pm

pytestmark = pytest.mark.gpu

FMTS = {"bf16": pm.MEM_KV_BF16, "fp8": pm.MEM_KV_FP8, "fp4": pm.MEM_KV_FP4}
FORMS = [pm.MEM_LATENT_ABSORBED, pm.MEM_LATENT_EXPANDED]


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    torch.cuda.synchronize()
    return t.float().cpu().numpy().astype(np.float64)


class Problem:
    """A seeded cache with `lens[i]` tokens in each chunk of request i, and queries over it.  What no request holds has
    all bits set: NaN in every format."""

    def __init__(self, seed, fmt, lens, nq, h, d, latent, page_tokens=32, ppc=2, k=None, docs=0, holes=False,
                 spread=1.0):
        rng = np.random.default_rng(seed)
        self.fmt, self.h, self.d, self.latent, self.T = fmt, h, d, latent, page_tokens
        m, flat = len(lens), [x for r in lens for x in r]
        n_chunks = len(flat) + 2
        n_pages = n_chunks * ppc + 2
        self.pool = np.full((n_pages, ref.page_bytes(fmt, page_tokens, latent)), 255, np.uint8)
        self.table = rng.permutation(n_pages)[:n_chunks * ppc].reshape(n_chunks, ppc).astype(np.int32)
        k = k or max(1, max(len(r) for r in lens))
        self.ids = np.full((m, k), -1, np.int32)
        self.tok_len = np.zeros(n_chunks, np.int32)
        self.chunk_ns = rng.integers(-1, docs, n_chunks).astype(np.int32) if docs else None
        order = rng.permutation(n_chunks)[:len(flat)]
        at = 0
        self.ctx = []                                       # per request: list of (page, row, chunk)
        for i, r in enumerate(lens):
            slots = np.sort(rng.permutation(k)[:len(r)]) if holes else np.arange(len(r))
            toks = []
            for s, n in zip(slots, r):
                c = order[at]
                at += 1
                self.ids[i, s] = c
                self.tok_len[c] = n
                t = np.arange(n)
                page, row = self.table[c, t // page_tokens], t % page_tokens
                toks += [(int(a), int(b), int(c)) for a, b in zip(page, row)]
                ref.put(fmt, page_tokens, self.pool, page, row, rng.standard_normal((n, latent)) * spread,
                        rng.standard_normal((n, ref.ROPE)) * spread)
            self.ctx.append(toks)
        if holes:
            for i in range(m):
                gone = self.ids[i] < 0
                self.ids[i, gone] = rng.choice([-1, n_chunks, 2 ** 31 - 1, -2 ** 31], gone.sum())
        self.nq = list(nq)
        self.off = np.concatenate([[0], np.cumsum(self.nq)]).astype(np.int32)
        total = int(self.off[-1])
        b16 = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16)  # noqa: E731
        self.q, self.t = b16(total, h, d), b16(total, h, ref.ROPE)
        self.w = (b16(h, 2 * d, latent).float() / np.sqrt(latent)).to(torch.bfloat16)
        self.query_ns = rng.integers(-1, docs, total).astype(np.int32) if docs else None
        self.scale = float(np.float32(1.0 / np.sqrt(d + ref.ROPE) / spread))

    def cache(self):
        return pm.LatentCache(up(self.pool), up(self.table), self.T, self.latent, ref.ROPE, self.fmt)

    def gpu(self, form, causal=False, window=0, prefix=None, q_pos=None, offsets=True, **kw):
        opt = lambda a: None if a is None else up(np.asarray(a, np.int32))  # noqa: E731
        q = kw.pop("q", None)
        lse = torch.full((len(self.q), self.h), 7.0, device="cuda")
        out = pm.mem_latent_attend(kw.pop("cache", None) or self.cache(), up(self.tok_len), up(self.ids),
                                   self.q.cuda() if q is None else q, kw.pop("t", self.t.cuda()),
                                   kw.pop("w", self.w.cuda()), self.scale, q_offsets=up(self.off) if offsets else None,
                                   q_pos=opt(q_pos), causal=causal, window=window, prefix_len=opt(prefix),
                                   chunk_ns=opt(self.chunk_ns), query_ns=opt(self.query_ns), form=form, lse=lse, **kw)
        return host(out), host(lse)

    def model(self, form, causal=False, window=0, prefix=None, q_pos=None):
        parts = []
        q, t, w = (x.float().numpy().astype(np.float64) for x in (self.q, self.t, self.w))
        for i, toks in enumerate(self.ctx):
            a, b = self.off[i], self.off[i + 1]
            n = len(toks)
            page, row = (np.array([x[j] for x in toks], np.int64) for j in (0, 1))
            present = (page >= 0) & (page < len(self.pool))
            c, r = ref.get(self.fmt, self.T, self.latent, self.pool, np.where(present, page, 0), row)
            c, r = np.where(present[:, None], c, 0), np.where(present[:, None], r, 0)
            doc = None if self.chunk_ns is None else np.array([self.chunk_ns[x] for _, _, x in toks], np.int64)
            qpos = np.arange(b - a) + n - (b - a) if q_pos is None else np.asarray(q_pos[a:b], np.int64)
            parts.append(ref.attend(form, q[a:b], t[a:b], c, r, w, doc, present, qpos,
                                    None if doc is None else self.query_ns[a:b], self.scale, causal, window,
                                    0 if prefix is None else prefix[i]))
        return [np.concatenate(x) for x in zip(*parts)]

    def check(self, name, forms=FORMS, offsets=True, **masks):
        for form in forms:
            out, lse = self.gpu(form, offsets=offsets, **masks)
            ref.check_attend(f"form {form}, {name}", out, lse, *self.model(form, **masks))


SHAPES = [("fp4", 16, 128, 512), ("fp4", 5, 64, 256), ("fp8", 12, 128, 512), ("fp8", 1, 64, 512), ("fp8", 33, 128, 256),
          ("bf16", 16, 128, 512), ("bf16", 3, 64, 256), ("bf16", 70, 64, 512)]


@pytest.mark.parametrize("name,h,d,latent", SHAPES)
def test_single_tokens(name, h, d, latent):
    # contexts of 0 tokens, 1 token, ends inside pages and units, chunks that hold nothing, holes in the lists
    lens = [[], [1], [64, 31, 64], [33], [0, 64, 0, 5], [64] * 7, [32], [2, 63, 64, 17, 1]]
    p = Problem(h + d, FMTS[name], lens, [1] * len(lens), h, d, latent, k=9, holes=True)
    p.check("plain", offsets=False)
    p.check("window", window=40)


@pytest.mark.parametrize("name,h,d,latent", SHAPES)
@pytest.mark.parametrize("masks", [dict(), dict(causal=True), dict(causal=True, window=37),
                                   dict(causal=True, window=9, prefix=[3, 0, 70, 1000, 5]), dict(window=1)])
def test_several_tokens(name, h, d, latent, masks):
    lens = [[64, 64, 20], [5], [64, 1, 64, 64], [40, 33], []]
    nq = [9, 5, 70, 0, 3]
    p = Problem(3 * h + d, FMTS[name], lens, nq, h, d, latent)
    p.check(str(masks), **masks)


@pytest.mark.parametrize("name,h,d,latent", SHAPES[:6:2] + SHAPES[6:])
def test_documents(name, h, d, latent):
    # chunks and tokens of three documents, deleted chunks, tokens that may see nothing
    lens = [[64, 20, 64, 1, 64], [64, 64], [3, 64, 9], []]
    p = Problem(h * d, FMTS[name], lens, [40, 1, 17, 2], h, d, latent, docs=3)
    p.check("documents")
    p.check("documents, causal", causal=True, prefix=[10, 0, 0, 0])
    p.check("documents, window", window=30)


@pytest.mark.parametrize("nq", [1, 2, 5, 16, 33, 64, 65, 128, 129, 200])
@pytest.mark.parametrize("h", [1, 3, 16])
def test_row_counts(nq, h):
    # rows (tokens x heads) around every tile's edge
    p = Problem(nq * h, FMTS["fp8"], [[64, 64, 64, 64], [64, 40]], [nq, nq], h, 64, 256)
    p.check("causal", causal=True, offsets=False)


def test_positions_of_new_tokens():
    lens, nq = [[64, 64], [30]], [6, 3]
    p = Problem(3, FMTS["fp8"], lens, nq, 4, 64, 256)
    q_pos = np.array([-5, 0, 127, 128, 2 ** 31 - 1, -2 ** 31, 3, 29, 30])
    for masks in (dict(causal=True), dict(causal=True, window=10), dict(window=2 ** 31 - 1)):
        p.check(str(masks), q_pos=q_pos, **masks)


def test_pages_outside_the_pool_keep_their_positions():
    p = Problem(8, FMTS["fp4"], [[64, 64, 64], [64, 50]], [5, 70], 4, 64, 256)
    p.table[p.ids[0, 1], 0], p.table[p.ids[1, 0], 1] = -1, len(p.pool)
    p.ctx = [[(int(p.table[c, i // 32]), i % 32, c) for c in map(int, p.ids[r][p.ids[r] >= 0])
              for i in range(p.tok_len[c])] for r in range(2)]
    p.check("plain")
    p.check("causal", causal=True, window=50)


@pytest.mark.parametrize("form", FORMS)
def test_rows_without_a_request_are_left_alone(form):
    p = Problem(5, FMTS["fp8"], [[64], [64, 9]], [3, 2], 4, 64, 256)
    total = 9                                               # two rows before the first request, two behind the last
    cache = p.cache()
    wide = lambda x: torch.cat([x[:2], x, x[:2]]).cuda()  # noqa: E731
    out = torch.full((total, 4, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    lse = torch.full((total, 4), 7.0, device="cuda")
    pm.mem_latent_attend(cache, up(p.tok_len), up(p.ids), wide(p.q), wide(p.t), p.w.cuda(), p.scale,
                         q_offsets=up(p.off + 2), form=form, out=out, lse=lse)
    got, gl = host(out), host(lse)
    assert (got[:2] == 7).all() and (got[7:] == 7).all() and (gl[:2] == 7).all() and (gl[7:] == 7).all()
    ref.check_attend("inside", got[2:7], gl[2:7], *p.model(form))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("name,where,value", [("bf16", "c", np.nan), ("bf16", "c", -np.inf), ("fp8", "c", np.nan),
                                              ("fp4", "c", np.nan), ("fp8", "r", np.inf), ("fp4", "r", np.nan)])
@pytest.mark.parametrize("nq", [6, 80])
def test_values_that_are_not_finite(form, name, where, value, nq):
    # they reach the rows that see them, all of those, and no other
    n = 160
    p = Problem(11, FMTS[name], [[64, 64, 32]], [nq], 3, 64, 256)
    clean = p.model(form, causal=True)
    at = n - nq + nq // 2                                   # seen by the later half of the new tokens
    page, row, _ = p.ctx[0][at]
    c, r = ref.get(p.fmt, p.T, p.latent, p.pool, page, row)
    (c if where == "c" else r)[5] = value
    ref.put(p.fmt, p.T, p.pool, page, row, c, r)
    out, lse = p.gpu(form, causal=True)
    sees = np.arange(nq) + n - nq >= at
    touched = np.repeat(sees[:, None], 3, 1)
    if value == np.inf:                                     # a key part at infinity: a score of -inf weighs nothing
        touched &= host(p.t)[:, :, 5] > 0
    assert not np.isfinite(out[touched]).any(), "rows that see it"
    assert np.isfinite(out[~touched]).all()
    ref.check_attend("others", out[~sees], lse[~sees], *[x[~sees] for x in clean])


@pytest.mark.parametrize("form", FORMS)
def test_odd_strides(form):
    p = Problem(21, FMTS["fp8"], [[64, 20], [33]], [4, 3], 5, 64, 256)
    want = p.gpu(form)
    total = 7
    flat = torch.zeros(total * 700 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(total, 700)
    fused = flat[:, :5 * 131].view(total, 5, 131)           # rows at odd elements
    q, t = fused[..., :64], fused[..., 65:129]
    q.copy_(p.q.cuda())
    t.copy_(p.t.cuda())
    major_q, major_t = (x.cuda().transpose(0, 1).contiguous().transpose(0, 1) for x in (p.q, p.t))
    w = torch.zeros((5, 136, 264), device="cuda", dtype=torch.bfloat16)[:, :128, :256]
    w.copy_(p.w.cuda())
    for kw in (dict(q=q, t=t), dict(q=major_q, t=major_t), dict(w=w)):
        got = p.gpu(form, **kw)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("spread", [1e-3, 40.0])
def test_small_and_large_scores(form, spread):
    # with large ones a token takes all the weight
    p = Problem(31, FMTS["bf16"], [[64, 64, 64]], [40], 3, 64, 256)
    p.scale *= spread
    p.check("scores", forms=[form], causal=True)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("m,nq,k", [(2, 1, 300), (1, 3, 700)])
def test_split_contexts(form, m, nq, k):
    # long lists of chunks: contexts that several workgroups share
    rng = np.random.default_rng(k)
    lens = [list(rng.integers(0, 65, k)) for _ in range(m)]
    p = Problem(k, FMTS["fp4"], lens, [nq] * m, 2, 64, 256)
    p.check("long", forms=[form], causal=True)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("h,nq,k", [(2, 1, 2600), (1, 5, 4096), (16, 9, 520), (16, 9, 4096)])
@pytest.mark.parametrize("latent", [256, 512])
def test_long_lists(form, h, nq, k, latent):
    # lists that leave a tile's other memory too little: other tiles
    rng = np.random.default_rng(k)
    p = Problem(k, FMTS["fp8"], [list(rng.integers(0, 3, 300)), [5]], [nq, nq], h, 64, latent, k=k, holes=True)
    p.check("long", forms=[form], causal=True)


@pytest.mark.parametrize("form", FORMS)
def test_many_ragged_requests(form):
    rng = np.random.default_rng(17)
    m = 600
    lens = [[int(x) for x in rng.integers(0, 40, rng.integers(0, 3))] for _ in range(m)]
    p = Problem(17, FMTS["fp8"], lens, rng.integers(0, 4, m), 2, 64, 256)
    p.check("ragged", forms=[form], causal=True)


@pytest.mark.parametrize("form", FORMS)
def test_repeated_calls_agree_and_graphs_replay(form):
    p = Problem(41, FMTS["fp8"], [[64] * 5, [64, 3]], [70, 2], 4, 64, 256)
    cache, total = p.cache(), 72
    q, t, w = p.q.cuda(), p.t.cuda(), p.w.cuda()
    args = (cache, up(p.tok_len), up(p.ids), q, t, w, p.scale)
    off = up(p.off)
    need = pm.mem_latent_attend_workspace_bytes(cache, 2, p.ids.shape[1], total, 4, 64, form)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    call = lambda: pm.mem_latent_attend(*args, q_offsets=off, causal=True, form=form, workspace=ws)  # noqa: E731
    first = call()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    graphs = []
    for _ in range(2):                                      # two graphs over one workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            graphs.append((g, call()))
        graphs[-1] = (g, graphs[-1][1])
    torch.cuda.synchronize()
    for seed in (1, 2, 3):
        q.copy_(torch.randn(q.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
        want = call().clone()
        assert torch.equal(call(), want)
        for g, out in graphs:
            ws.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
    assert first.shape == (total, 4, 64)


def test_empty_calls():
    p = Problem(1, FMTS["fp4"], [[5]], [1], 2, 64, 256)
    x = torch.zeros((0, 2, 128), device="cuda", dtype=torch.bfloat16)
    for form in FORMS:
        out = pm.mem_latent_attend(p.cache(), up(p.tok_len), up(p.ids), x[..., :64], x[..., 64:], p.w.cuda(), 1.0,
                                   form=form)
        assert out.shape == (0, 2, 64)
