"""The attention's main loops over many units per workgroup (contexts that are
not split), and large cache calls over rows that 16-byte accesses cannot reach."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2607_05708_amd as pm
from test_gpu_kv import FMTS, host, new_cache, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Shared:
    """m requests over the same chunks of one key/value head, each in an order of its own: enough workgroups that
    contexts are not split, so that each walks all of its units, 128 or 256 at a time (BATCH)."""

    def __init__(self, seed, fmt, d, m, nq, group, n_chunks, page_tokens=32, ragged=False, docs=False):
        rng = np.random.default_rng(seed)
        self.fmt, self.d, self.m, self.nq, self.group, self.T = fmt, d, m, nq, group, page_tokens
        self.rng, self.docs = rng, docs
        self.pool, self.table = new_cache(fmt, n_chunks, 1, page_tokens, 1, d, seed)
        self.tok = np.full(n_chunks, page_tokens, np.int32)
        if ragged:
            self.tok[rng.permutation(n_chunks)[:n_chunks // 3]] = rng.integers(1, page_tokens, n_chunks // 3)
        self.ns = (np.arange(n_chunks) % 2).astype(np.int32)
        x = rng.standard_normal((2, n_chunks * page_tokens, 1, d))
        chunk, pos = np.repeat(np.arange(n_chunks), page_tokens), np.tile(np.arange(page_tokens), n_chunks)
        ref.put(fmt, page_tokens, self.pool, self.table[chunk, 0], pos, x[0], x[1])
        self.k, self.v = (y.reshape(n_chunks, page_tokens, 1, d) for y in
                          ref.get(fmt, page_tokens, 1, d, self.pool, self.table[chunk, 0], pos))
        self.ids = np.stack([np.roll(np.arange(n_chunks), 7 * i) for i in range(m)]).astype(np.int32)
        self.q = torch.from_numpy(rng.standard_normal((m * nq, group, d)).astype(np.float32)).to(torch.bfloat16)
        self.query_ns = (np.arange(m * nq) % 2).astype(np.int32)  # neighbours differ: every unit is masked
        self.scale = float(np.float32(1.0 / np.sqrt(d)))
        self.cache = pm.KvCache(up(self.pool), up(self.table), page_tokens, 1, d, fmt)
        self.args = up(self.tok), up(self.ids), self.q.cuda()
        self.doc_args = dict(chunk_ns=up(self.ns), query_ns=up(self.query_ns)) if docs else {}
        # contexts are not split
        assert pm.mem_attend_workspace_bytes(self.cache, m, n_chunks, m * nq, group) == 0

    def gpu(self, **masks):
        out, lse = pm.mem_attend(self.cache, *self.args, self.scale, **self.doc_args, **masks)
        return host(out).reshape(self.m, self.nq, self.group, self.d), host(lse).reshape(self.m, self.nq, self.group)

    def check(self, name, out, lse, i, **masks):
        """Request i's first and last tokens, with the first and last heads, against the 64-bit model."""
        own = self.ids[i]
        k, v = (np.concatenate([y[c, :self.tok[c]] for c in own]) for y in (self.k, self.v))
        doc = np.repeat(self.ns[own], self.tok[own]) if self.docs else None
        n, at, heads = len(k), np.unique([0, self.nq - 1]), np.unique([0, self.group - 1])
        q = self.q.float().numpy().astype(np.float64)[i * self.nq + at][:, heads]
        want = ref.attend(q, k, v, doc, np.ones(n, bool), at + n - self.nq,
                          self.query_ns[i * self.nq + at] if self.docs else None, self.scale,
                          masks.get("causal", False), masks.get("window", 0), 0, masks.get("softcap", 0.0), None)
        ref.check_attend(f"{name}, request {i}", out[i][at][:, heads], lse[i][at][:, heads], *want)

    def put_value(self, unit, at, bits):
        """NaN as the last element of the value of token `at` of a chunk (in 8 bits by its code or, as in 4, its scale);
        returns what takes it back."""
        page = self.cache.pool[int(self.table[unit, 0])]
        r, s = ref.row_bytes(self.fmt, self.d)
        codes, scales = self.T * r + at * r, 2 * self.T * r + self.T * s + at * s
        old = page.clone()
        if self.fmt == ref.BF16:
            page[codes + r - 2:codes + r] = torch.tensor(bits, dtype=torch.uint8, device="cuda")
        elif self.fmt == ref.FP8 and bits[0] == 0x81:
            page[codes + r - 1] = 0x7F
        else:
            page[scales + s - 1] = 255
        return lambda: page.copy_(old)


# tokens a request, heads of its group, requests: rounds of workgroups that fill the GPU as they are
TILES = [("fp4", 64, 8, 16, 768), ("fp8", 64, 43, 3, 768), ("bf16", 64, 8, 16, 768), ("fp4", 128, 8, 16, 512),
         ("fp8", 128, 16, 8, 512), ("bf16", 128, 8, 16, 512), ("fp4", 256, 8, 16, 256), ("fp8", 256, 8, 16, 256),
         ("bf16", 256, 8, 16, 256)]
FEW16 = [("fp4", 64, 4, 4, 1536), ("fp8", 128, 2, 8, 1536), ("bf16", 128, 1, 16, 1536), ("fp4", 256, 3, 5, 512)]
FEW32 = [("fp4", 64, 2, 16, 1536), ("fp8", 128, 8, 4, 1024), ("bf16", 256, 2, 16, 512), ("fp4", 128, 16, 4, 1024)]
MASKS = [dict(), dict(causal=True), dict(causal=True, window=6000), dict(causal=True, softcap=20.0),
         dict(causal=True, window=5000, softcap=1e4)]


@pytest.mark.parametrize("masks", MASKS)
@pytest.mark.parametrize("name,d,nq,group,m,units", [(*t, 273) for t in TILES] + [(*t, 571) for t in FEW16 + FEW32])
def test_contexts_of_several_batches_of_units(name, d, nq, group, m, units, masks):
    # 273 units are three batches of tiles of 128 rows and 137 steps, 571 three batches of the others
    p = Shared(d + nq, FMTS[name], d, m, nq, group, units, ragged=True)
    out, lse = p.gpu(**masks)
    for i in (0, m // 2 + 1):
        p.check("batches", out, lse, i, **masks)


@pytest.mark.parametrize("name,d,nq,group,m,units,batch",
                         [(*t, 273, 128) for t in (TILES[0], TILES[1], TILES[3], TILES[5], TILES[7])] +
                         [(*t, 571, 256) for t in (FEW16[1], FEW32[0], FEW32[2])])
def test_values_that_are_not_finite_wherever_their_unit_stands(name, d, nq, group, m, units, batch):
    # Rows of two documents by turns, so that every unit is masked.  A value of NaN, at each place of a step, of the
    # steps that share what is noted of them, and at both sides of a batch's edge, shows in the rows of its document,
    # and the others are what they were, bit for bit.
    p = Shared(3 * d, FMTS[name], d, m, nq, group, units, docs=True)
    clean = p.gpu()
    p.check("clean", *clean, 0)
    doc = p.query_ns.reshape(m, nq)
    for back in [0, 1, 2, 3, 4, 5, 6, 7, batch - 2, batch - 1, batch, batch + 1, batch + 2, 2 * batch - 1, 2 * batch]:
        unit = int(p.ids[0][units - 1 - back])               # `back` units before the end of request 0
        undo = p.put_value(unit, (5 * back) % 32, (0xC0, 0x7F) if back % 2 else (0x81, 0x7F))
        out, lse = p.gpu()
        undo()
        sees = doc == p.ns[unit]
        assert np.isnan(out[sees][..., -1]).all(), f"{back} units from the end"
        assert np.array_equal(out[~sees], clean[0][~sees]) and np.array_equal(lse, clean[1])


@pytest.mark.parametrize("name,d,nq,group,m,units", [(*t, 273) for t in (TILES[1], TILES[5])] + [(*FEW16[2], 571)])
def test_a_value_that_is_not_finite_behind_long_runs_without_a_mask(name, d, nq, group, m, units):
    # masked units at the end and at the window's edge only
    p = Shared(5 * d, FMTS[name], d, m, nq, group, units)
    masks = dict(causal=True, window=32 * units - 300)
    clean = p.gpu(**masks)
    p.check("clean", *clean, 0, **masks)
    total = 32 * units
    at = total - nq + np.arange(nq)                          # positions of the new tokens
    for pos in (total - 1, total - 2, total - 40, total // 2, 301, 300 - nq // 2, 299 - nq, 100):
        unit = int(p.ids[0][pos // 32])
        undo = p.put_value(unit, pos % 32, (0xC0, 0x7F))
        out, lse = p.gpu(**masks)
        undo()
        sees = (pos <= at) & (pos > at - masks["window"])
        assert np.isnan(out[0][sees][..., -1]).all(), pos
        assert np.array_equal(out[0][~sees], clean[0][0][~sees]) and np.array_equal(lse, clean[1])


@pytest.mark.parametrize("name", list(FMTS))
@pytest.mark.parametrize("heads,d,n", [(3, 64, 44001), (5, 128, 14003), (1, 256, 33003)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_calls_over_strided_rows(name, heads, d, n, dtype):
    # several items a thread: rows at odd elements and views of a fused projection do what contiguous rows do
    fmt, T = FMTS[name], 64
    pool, table = new_cache(fmt, -(-n // 128), 2, T, heads, d)
    at = np.random.default_rng(n).permutation(len(table) * 128)[:n]
    chunk, pos = (at // 128).astype(np.int32), (at % 128).astype(np.int32)
    chunk[::777] = -1
    where = up(chunk), up(pos)

    def odd(t):                                              # rows of d + 1 elements, tokens 3 elements apart
        return t[1:].view(n, heads * (d + 1) + 3)[:, :heads * (d + 1)].view(n, heads, d + 1)[:, :, :d]

    g = torch.Generator("cuda").manual_seed(n)
    flat = torch.randn(n * (heads * (d + 1) + 3) + 1, device="cuda", generator=g).to(dtype)
    fused = torch.randn((n, 2 * heads + 1, d), device="cuda", generator=g).to(dtype)
    for k, v in ((odd(flat), fused[:, 1:1 + heads]), (fused[:, 1:1 + heads], fused[:, 1 + heads:])):
        caches = [pm.KvCache(up(pool), up(table), T, heads, d, fmt) for _ in range(2)]
        pm.mem_kv_write(caches[0], k, v, *where)
        pm.mem_kv_write(caches[1], k.contiguous(), v.contiguous(), *where)
        assert torch.equal(caches[0].pool, caches[1].pool)
        want = pm.mem_kv_read(caches[0], *where, dtype=dtype)
        out, both = torch.full_like(flat, 7.0), torch.full((n, 2, heads, d), 7.0, device="cuda", dtype=dtype)
        for pair in ((odd(out), both[:, 1]), (both[:, 0], both[:, 1])):
            pm.mem_kv_read(caches[0], *where, out=pair)
            assert all(torch.equal(a, b) for a, b in zip(pair, want))
        gaps = torch.ones_like(flat, dtype=torch.bool)
        odd(gaps).fill_(False)
        assert (out[gaps] == 7).all()
