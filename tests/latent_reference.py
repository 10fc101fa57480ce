"""Plain 64-bit model of the rotation, the latent cache and the attention over it,
from the formulas of include/memattn_append.h and include/memattn_latent.h, in
numpy."""
import numpy as np

import kv_reference as kv

ROPE = 64


def rotate(x, at, freq, pairs):
    """Rows [n, ..., d] rotated by the positions `at` [n], in 64 bits."""
    x = np.array(x, np.float64)
    half = len(freq)
    t = np.asarray(at, np.float64)[:, None] * np.asarray(freq, np.float64)
    t = t.reshape(len(x), *[1] * (x.ndim - 2), half)
    lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    with np.errstate(invalid="ignore"):
        a, b = x[..., lo].copy(), x[..., hi].copy()
        x[..., lo] = a * np.cos(t) - b * np.sin(t)
        x[..., hi] = a * np.sin(t) + b * np.cos(t)
    return x


def page_bytes(fmt, page_tokens, latent):
    r, s = kv.row_bytes(fmt, latent)
    return page_tokens * (r + 2 * ROPE + s)


def views(fmt, page_tokens, latent, pool):
    """(codes, key parts, scales) of a pool uint8 [pages, page_bytes]: [pages, row, bytes]."""
    r, s = kv.row_bytes(fmt, latent)
    t = page_tokens

    def view(offset, width):
        return np.lib.stride_tricks.as_strided(pool[:, offset:], (len(pool), t, width), (pool.strides[0], width, 1))

    scales = view(t * (r + 2 * ROPE), s) if s else np.zeros((len(pool), t, 0), np.uint8)
    return view(0, r), view(t * r, 2 * ROPE), scales


def put(fmt, page_tokens, pool, page, row, c, r):
    """Store tokens' rows c [..., latent] and r [..., ROPE] at (page, row) of the pool."""
    codes, parts, scales = views(fmt, page_tokens, c.shape[-1], pool)
    codes[page, row], scales[page, row] = kv.encode_rows(fmt, c)
    parts[page, row] = kv.encode_rows(kv.BF16, r)[0]


def get(fmt, page_tokens, latent, pool, page, row):
    """Tokens' (c, r) rows, float64."""
    codes, parts, scales = views(fmt, page_tokens, latent, pool)
    return (kv.decode_rows(fmt, codes[page, row], scales[page, row]),
            kv.decode_rows(kv.BF16, parts[page, row], scales[page, row][..., :0]))


ABSORBED, EXPANDED = 1, 2
SIX = 6.0  # Hoeffding: a sum of errors of at most a_i each leaves +- 6 sqrt(sum a_i^2) once in 3e7


def attend(form, q, t, c, r, w, doc, present, qpos, qdoc, scale, causal, window, prefix):
    """One request in float64, with the form's roundings of W^T q, or of keys and values, to bf16: q [nq, h, d], t [nq,
    h, ROPE]; c [n, latent], r [n, ROPE]; w [h, 2 d, latent]; doc [n] or None; present [n].  Returns out [nq, h, d], lse
    [nq, h], and what a kernel may differ by in each.

    A score: fp32 sums in some order; where such a sum lands on the other side of a rounding border, an element of W^T
    q or of the key is one step off, 2^-7 of itself at most: two such elements are allowed for.  A score that is off by
    e changes a weight by a factor of e^(2 e) at most.  Weights are rounded to bf16, 2^-8 of themselves at most; in the
    absorbed form the weighted sum of latent vectors is too.  These errors are many and independent (Hoeffding).  The
    output's own rounding: 2^-8 of it.  fp32 sums stay below 2^-14 of the magnitudes for the lengths used here."""
    nq, h, d = q.shape
    n = len(c)
    out, tol = np.zeros((nq, h, d)), np.zeros((nq, h, d))
    lse, tol_l = np.full((nq, h), -np.inf), np.zeros((nq, h))
    p = np.arange(n)
    for x in range(h):
        wk, wv = w[x, :d], w[x, d:]
        keys, vals, ql = c @ wk.T, c @ wv.T, q[:, x] @ wk
        if form == ABSORBED:
            left, right = kv.to_bf16(ql), c
        else:
            left, right, vals = q[:, x], kv.to_bf16(keys), kv.to_bf16(vals)
        s = scale * (left @ right.T + t[:, x] @ r.T)
        sums = scale * (np.abs(left) @ np.abs(right).T + np.abs(t[:, x]) @ np.abs(r).T)
        for j in range(nq):
            see = present.copy()
            rule = np.ones(n, bool)
            if causal:
                rule &= p <= qpos[j]
            if window:
                rule &= p > qpos[j] - window
            see &= rule | (p < prefix)
            if doc is not None:
                see &= (doc >= 0) & (doc == qdoc[j])
            if not see.any():
                continue
            e = sums[j, see] * (left.shape[1] + ROPE) * 2.0 ** -24 + np.abs(s[j, see]) * 2.0 ** -21
            e = (e + 2 * 2.0 ** -7 * scale * np.abs(left[j] * right[see]).max(1)).max() + 2.0 ** -20
            z, v = s[j, see], vals[see]
            top = z.max()
            u = np.exp(z - top)
            u /= u.sum()
            out[j, x] = u @ v
            lse[j, x] = top + np.log(np.exp(z - top).sum())
            size = u @ np.abs(v)
            b = np.expm1(2 * e) * size + size * 2.0 ** -14 + 2.0 ** -8 * np.abs(out[j, x])
            b += np.minimum(2.0 ** -8 * size, SIX * 2.0 ** -8 * np.sqrt(np.square(u[:, None] * v).sum(0)))
            if form == ABSORBED:
                o = u @ c[see]
                b += np.minimum(2.0 ** -8 * (np.abs(wv) @ np.abs(o)), SIX * 2.0 ** -8 * np.sqrt(np.square(wv * o).sum(1)))
            else:
                b += 2 * 2.0 ** -7 * (u[:, None] * np.abs(v)).max(0)
            tol[j, x], tol_l[j, x] = b, e + see.sum() * 2.0 ** -24 + np.abs(lse[j, x]) * 2.0 ** -21
    return out, lse, tol, tol_l


def check_attend(name, got_out, got_lse, out, lse, tol, tol_l):
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got_lse), empty), f"{name}: rows without a visible token"
    assert np.all(got_out[empty] == 0), f"{name}: rows without a visible token are not zero"
    off = np.where(empty[..., None], 0, np.abs(got_out - out))
    bad = ~(off <= tol + 1e-30)
    assert not bad.any(), (f"{name}: {bad.sum()} of {bad.size} outputs off, worst "
                           f"{np.nanmax(off / (tol + 1e-30)):.3g} tolerances, first {np.argwhere(bad)[0]}")
    off = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, lse))
    bad = ~(off <= tol_l)
    assert not bad.any(), f"{name}: {bad.sum()} lse off, worst {np.nanmax(off):.3g}"
