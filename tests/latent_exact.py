"""Latent attention whose scores are exact, so that what is left to be off is known closely.

Element 0 of a query is the only one that is not 0, and row 0 of W_h is 1 in one column: W_h^T q and that element of the
keys are exact in bf16.  One element of the key parts counts, in steps of 1/8.  A score is the sum of two numbers of few
bits: exact in fp32."""
import numpy as np
import torch

import kv_reference as kv
import latent_reference as ref
from test_gpu_latent import Problem

SIX = ref.SIX
ABSORBED, EXPANDED = ref.ABSORBED, ref.EXPANDED
HALF = 2.0 ** -8    # of a bf16 number: the most that rounding to it moves


def tile_rows(form, m, total_q, h):
    """Rows of the tiles that a call with a short list takes."""
    if form == EXPANDED:
        return 128
    return 16 if total_q * h <= 32 * m else 64 if total_q * h <= 64 * m else 128


class Exact(Problem):
    def __init__(self, seed, fmt, lens, nq, h, d, latent, even=False, **kw):
        super().__init__(seed, fmt, lens, nq, h, d, latent, **kw)
        rng = np.random.default_rng(seed + 1)
        total = len(self.q)
        pick = lambda *s: torch.from_numpy(rng.choice([0.5, 1.0, 2.0], s)).to(torch.bfloat16)  # noqa: E731
        self.q.zero_()
        self.t.zero_()
        if not even:                                        # even: all scores are 0
            self.q[..., 0], self.t[..., 0] = pick(total, h), pick(total, h)
        self.column = rng.integers(0, latent, h)
        self.w[:, 0] = 0
        for x in range(h):
            self.w[x, 0, self.column[x]] = 1
        _, parts, _ = ref.views(self.fmt, self.T, latent, self.pool)
        steps = np.zeros((*parts.shape[:2], ref.ROPE))
        steps[..., 0] = rng.integers(-8, 9, parts.shape[:2]) / 8
        steps[..., 1:] = rng.standard_normal((*parts.shape[:2], ref.ROPE - 1))
        parts[...] = kv.encode_rows(kv.BF16, steps)[0]
        self.scale = 1.0

    def tokens(self, i):
        """(c, r) of request i's context."""
        page, row = (np.array([x[j] for x in self.ctx[i]], np.int64) for j in (0, 1))
        return ref.get(self.fmt, self.T, self.latent, self.pool, page, row)

    def row(self, form, rows, i, j, x, see, c, r, one_sum=False, one_weight=False):
        """Of token j (of all) and head x over the tokens `see` of request i: out [d], lse, and what a kernel with tiles of
        `rows` rows may differ by in each.  one_sum, one_weight: a mistake, sums or weights rounded to one bf16.

        fp32: weights are off by 2^-19 of themselves at most (the score times log2(e), the exponential), and a sum of n
        terms in chains of n / 2 by n 2^-25.  Sums go through V_h, and the weights of tiles of 16 rows to the sums, as two
        bf16 numbers: 2^-17 of each at most, those of the sums many and independent (Hoeffding); products with V_h in
        fp32, in chains of 64: 2^-18 of their magnitudes.  Other weights are rounded to bf16, many and independent, and
        so are values in the expanded form, where an fp32 sum on the other side of a border moves one by a step (less than
        one in 3,000: more than four where the context is short, once in 10^7).  The output's own rounding."""
        wv = self.w[x, self.d:].double().numpy()
        s = float(self.q[j, x, 0]) * c[see, self.column[x]] + float(self.t[j, x, 0]) * r[see, 0]
        top = s.max()
        u = np.exp(s - top)
        lse = top + np.log(u.sum())
        w = kv.to_bf16(u) if one_weight else u
        u, w = u / u.sum(), w / u.sum()
        n = len(s)
        if form == ABSORBED:
            v = c[see] @ wv.T
            o = w @ c[see]
            out = wv @ (kv.to_bf16(o) if one_sum else o)
            size = u @ np.abs(v)
            tol = SIX * 2.0 ** -17 * np.sqrt(np.square(wv * o).sum(1)) + 2.0 ** -18 * (np.abs(wv) @ np.abs(o))
        else:
            v = kv.to_bf16(c[see] @ wv.T)
            out, size = w @ v, u @ np.abs(v)
            tol = (4 + n / 300) * 2.0 ** -7 * (u[:, None] * np.abs(v)).max(0)
        tol = tol + size * (2.0 ** -18 + 2.0 ** -17 + n * 2.0 ** -25) + HALF * np.abs(out)
        if rows > 16 and np.ptp(s):
            off = np.sqrt(np.square(u[:, None] * (v - out)).sum(0))
            tol = tol + np.minimum(SIX * HALF * off, 2 * HALF * size) * (1 + HALF)
        return out, lse, tol, 2.0 ** -18 + n * 2.0 ** -25 + abs(lse) * 2.0 ** -22

    def sees(self, i, pos, causal=False, window=0):
        p = np.arange(len(self.ctx[i]))
        return ((p <= pos) if causal else p >= 0) & ((p > pos - window) if window else p >= 0)

    def check_rows(self, form, sample, out, lse, q_pos=None, **masks):
        """Rows (request, token of all, head) against the model."""
        rows = tile_rows(form, len(self.nq), len(self.q), self.h)
        worst, kept = 0.0, {}
        for i, j, x in sample:
            if id(self.ctx[i]) not in kept:
                kept[id(self.ctx[i])] = self.tokens(i)
            c, r = kept[id(self.ctx[i])]
            pos = len(c) - self.nq[i] + j - self.off[i] if q_pos is None else q_pos[j]
            want, l, tol, tol_l = self.row(form, rows, i, j, x, self.sees(i, pos, **masks), c, r)
            off = np.abs(out[j, x] - want) / tol
            worst = max(worst, off.max(), abs(lse[j, x] - l) / tol_l)
            assert off.max() <= 1, f"form {form}, request {i}, token {j}, head {x}: {off.max():.3g} tolerances"
            assert abs(lse[j, x] - l) <= tol_l, f"form {form}, token {j}, head {x}: lse {lse[j, x]}, not {l}"
        return worst
