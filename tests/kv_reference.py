"""Plain 64-bit model of the key/value cache and of attention over it, from the
formulas of include/memattn_kv.h, in numpy."""
import numpy as np

BF16, FP8, FP4 = 0, 1, 2
BLOCK = 32
TOP = {FP8: 464.0, FP4: 7.0}
E_MAX = {FP8: 119, FP4: 125}


def _grid(fmt):
    """Non-negative values of codes 0, 1, ... of a format."""
    if fmt == FP4:
        return np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
    vals = []
    for c in range(127):
        ex, man = c >> 3, c & 7
        vals.append(man / 8 * 2.0 ** -6 if ex == 0 else (1 + man / 8) * 2.0 ** (ex - 7))
    return np.array(vals)


GRID = {FP8: _grid(FP8), FP4: _grid(FP4)}


def to_bf16(x):
    """float64 values rounded to bf16 (nearest, ties to even)."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        man, ex = np.frexp(x)
        step = np.ldexp(1.0, np.maximum(ex - 8, -133))
        r = np.round(x / step) * step
    return np.where(np.isfinite(x), r, x)


def bf16_bits(x):
    u = np.asarray(x, np.float32).view(np.uint32)
    assert np.all((u & 0xFFFF) == 0) or np.isnan(x).any()
    return (u >> 16).astype(np.uint16)


def scale_exponent(fmt, a):
    """Smallest e with a <= TOP * 2^e, clamped, for each magnitude."""
    a = np.asarray(a, np.float64)
    e = np.floor(np.log2(np.maximum(a, 1e-60) / TOP[fmt])).astype(np.int64) - 1
    for _ in range(4):
        e = e + (a > np.ldexp(TOP[fmt], e))
    return np.clip(e, -110, E_MAX[fmt])


def encode_rows(fmt, x):
    """(codes uint8 [..., bytes], scale bytes uint8 [..., d / 32]) of float rows [..., d]."""
    x = np.asarray(x, np.float64)
    if fmt == BF16:
        bits = bf16_bits(to_bf16(x))
        return np.ascontiguousarray(bits).view(np.uint8), np.zeros((*x.shape[:-1], 0), np.uint8)
    b = x.reshape(-1, BLOCK)
    nan = np.isnan(b).any(1)
    sign = np.signbit(b)
    big = float(np.finfo(np.float32).max)
    mag = np.minimum(np.abs(np.where(nan[:, None], 0.0, b)), big)
    e = scale_exponent(fmt, mag.max(1))
    grid = GRID[fmt]
    y = np.minimum(np.ldexp(mag, -e[:, None]), grid[-1])
    hi = np.clip(np.searchsorted(grid, y), 1, len(grid) - 1)
    lo = hi - 1
    above, below = grid[hi] - y, y - grid[lo]
    c = np.where(above < below, hi, np.where(below < above, lo, np.where(hi % 2 == 0, hi, lo)))
    codes = (c + np.where(sign, 128 if fmt == FP8 else 8, 0)).astype(np.uint8)
    codes[nan] = 0                             # a NaN block's codes say nothing
    codes = codes.reshape(x.shape)
    if fmt == FP4:
        codes = codes[..., 0::2] | (codes[..., 1::2] << 4)
    scale = np.where(nan, 255, e + 127).astype(np.uint8)
    return codes, scale.reshape(*x.shape[:-1], x.shape[-1] // BLOCK)


def decode_rows(fmt, codes, scale):
    """float64 rows of codes and scale bytes."""
    codes = np.ascontiguousarray(codes)
    if fmt == BF16:
        return (codes.view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    if fmt == FP4:
        c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
        v = GRID[FP4][c & 7] * np.where(c & 8, -1.0, 1.0)
    else:
        mag = np.append(GRID[FP8], np.nan)
        v = mag[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, -1)


def row_bytes(fmt, d):
    return {BF16: (2 * d, 0), FP8: (d, d // BLOCK), FP4: (d // 2, d // BLOCK)}[fmt]


def page_bytes(fmt, page_tokens, heads, d):
    r, s = row_bytes(fmt, d)
    return heads * 2 * page_tokens * (r + s)


def views(fmt, page_tokens, heads, d, pool):
    """((K codes, K scales), (V codes, V scales)) of a pool uint8 [pages, page_bytes]: [pages, heads, row, bytes]."""
    r, s = row_bytes(fmt, d)
    t = page_tokens

    def view(offset, width):
        return np.lib.stride_tricks.as_strided(pool[:, offset:], (len(pool), heads, t, width),
                                               (pool.strides[0], 2 * t * (r + s), width, 1))

    codes = [view(w * t * r, r) for w in (0, 1)]
    scales = [view(2 * t * r + w * t * s, s) if s else np.zeros((len(pool), heads, t, 0), np.uint8) for w in (0, 1)]
    return list(zip(codes, scales))


def put(fmt, page_tokens, pool, page, row, k, v):
    """Store tokens' rows [..., heads, d] at (page, row) (numbers or arrays) of the pool."""
    for (codes, scales), x in zip(views(fmt, page_tokens, k.shape[-2], k.shape[-1], pool), (k, v)):
        c, s = encode_rows(fmt, x)
        codes[page, :, row] = c
        scales[page, :, row] = s


def get(fmt, page_tokens, heads, d, pool, page, row):
    """Tokens' (k, v) rows, float64 [..., heads, d]."""
    return [decode_rows(fmt, codes[page, :, row], scales[page, :, row])
            for codes, scales in views(fmt, page_tokens, heads, d, pool)]


def attend(q, k, v, doc, present, qpos, qdoc, scale, causal, window, prefix, cap, slopes):
    """One request in float64: q [nq, hq, d]; k, v [n, h, d]; doc [n] or None; present [n].  Returns out [nq, hq, d],
    lse [nq, hq], and for each row the bounds that an fp32 / bf16 kernel's error follows from: the weighted sum of
    |v| and the largest error of a visible score."""
    nq, hq, d = q.shape
    n, h = k.shape[0], k.shape[1]
    out, mag = np.zeros((nq, hq, d)), np.zeros((nq, hq, d))
    lse, err = np.full((nq, hq), -np.inf), np.zeros((nq, hq))
    p = np.arange(n)
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
        for x in range(hq):
            kk, vv = k[see, x // (hq // h)], v[see, x // (hq // h)]
            s = scale * (kk @ q[j, x])
            # fp32 products and sums in some order, then a few roundings of the score itself
            e = scale * (np.abs(kk) @ np.abs(q[j, x])) * d * 2.0 ** -24 + np.abs(s) * 2.0 ** -21
            if cap:
                s = cap * np.tanh(s / cap)
                e = e + cap * 2.0 ** -20
            if slopes is not None:
                bias = slopes[x] * np.abs(qpos[j] - p[see])
                s = s - bias
                e = e + (bias + np.abs(s)) * 2.0 ** -21
            top = s.max()
            w = np.exp(s - top)
            out[j, x] = (w @ vv) / w.sum()
            mag[j, x] = (w @ np.abs(vv)) / w.sum()
            lse[j, x] = top + np.log(w.sum())
            err[j, x] = e.max() + see.sum() * 2.0 ** -24 + 2.0 ** -20
    return out, lse, mag, err


def check_attend(name, got_out, got_lse, out, lse, mag, err):
    """Compare a kernel's outputs with the model's.  A weight rounded to bf16 is off by some 2^-9 of itself (half an
    ulp is 2^-8 at most), which division by the rounded weights' sum partly cancels: 2^-9 of the weighted |v| is
    allowed for; the output's own rounding adds at most 2^-8 of it; a score that is off by e moves weights by
    2 e; fp32 sums of the products stay below 2^-14 of the weighted |v| for the lengths used here."""
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got_lse), empty), f"{name}: rows without a visible token"
    assert np.all(got_out[empty] == 0), f"{name}: rows without a visible token are not zero"
    e = err[..., None]
    tol = mag * (2.0 ** -9 + 2.0 ** -14 + 2 * e) + np.abs(out) * 2.0 ** -8 + 1e-30
    bad = ~(np.abs(got_out - out) <= tol) & ~empty[..., None]
    assert not bad.any(), (f"{name}: {bad.sum()} of {bad.size} outputs off, worst "
                           f"{np.nanmax(np.abs(got_out - out) / tol):.3g} tolerances, first {np.argwhere(bad)[0]}")
    live = ~empty
    tol_l = err + np.abs(np.where(live, lse, 0)) * 2.0 ** -21
    bad = ~(np.abs(np.where(live, got_lse - np.where(live, lse, 0), 0)) <= tol_l)
    assert not bad.any(), f"{name}: {bad.sum()} lse off, worst {np.abs(got_lse - lse)[live].max():.3g}"
