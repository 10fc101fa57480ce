"""Capped scores over the whole range of caps: a cap far above the scores leaves
them as they are, and the error of a capped score goes with the score."""
import numpy as np
import pytest
import torch

import kv_reference as ref
from test_gpu_kv import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def model(p, cap, bias=False, **masks):
    """The 64-bit model with bounds that do not grow with the cap.  The tanh never stretches the error that a raw score
    brings with it.  Its own: 1 - 2 / (1 + e^2x), with an exponential, a sum and a reciprocal that are each off by an ulp
    at most (2^-23 of themselves), is off by 2^-21, or 2^-22 where |x| is above 0.1875, which is 2^-19 of a tanh of at
    least 0.185; below that a series is off by less.  With caps of up to 64 the first may stand for all scores."""
    out, lse, mag, _ = p.model(cap=cap, bias=bias, **masks)
    _, _, _, err = p.model(bias=bias, **masks)
    top = np.zeros_like(err)
    q = p.q.float().numpy().astype(np.float64)
    for i, toks in enumerate(p.ctx):
        if not toks:
            continue
        page, row = (np.array([t[j] for t in toks], np.int64) for j in (0, 1))
        k, _ = ref.get(p.fmt, p.T, p.heads, p.d, p.pool, page, row)
        for j in range(p.off[i], p.off[i + 1]):
            for h in range(p.hq):
                top[j, h] = np.abs(p.scale * (k[:, h // (p.hq // p.heads)] @ q[j, h])).max()
    return out, lse, mag, err + np.minimum(top, cap) * 2.0 ** -19 + (cap * 2.0 ** -21 if cap <= 64 else 0.0)


CAPS = [5.0, 30.0, 64.0, 65.0, 1e3, 1e4, 1e5, 1e6, 1e8, 1e19, 1e30, 3e38]
SHAPES = [("fp4", 4, 1, 128), ("fp8", 3, 3, 64), ("bf16", 2, 1, 256)]


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("nq", [1, 6, 20, 90])
@pytest.mark.parametrize("name,hq,heads,d", SHAPES)
def test_caps_of_every_size(name, hq, heads, d, nq, cap):
    # units that every row sees whole, units with a mask, units with a bias
    p = Problem(nq + d, dict(fp4=ref.FP4, fp8=ref.FP8, bf16=ref.BF16)[name], [[64, 64, 64, 31]], [nq], hq, heads, d)
    for masks in (dict(), dict(causal=True, window=50), dict(bias=True), dict(causal=True, bias=True, window=70)):
        out, lse = p.gpu(cap=cap, **masks)
        ref.check_attend(f"{masks}", out, lse, *model(p, cap, **masks))


@pytest.mark.parametrize("nq", [2, 12, 90])
@pytest.mark.parametrize("cap", [1e3, 1e5, 1e7])
def test_a_row_of_large_scores_beside_small_ones(nq, cap):
    # one token's scores are of the cap's size, its neighbours' are not
    p = Problem(nq, ref.FP8, [[64, 64, 40]], [nq], 4, 2, 128)
    big = nq // 2
    p.q[big] *= cap
    small = np.arange(nq) != big
    for masks in (dict(), dict(causal=True)):
        got, want = p.gpu(cap=cap, **masks), model(p, cap, **masks)
        ref.check_attend(f"{masks}", *[x[small] for x in (*got, *want)])
        assert np.isfinite(got[0]).all() and (np.abs(got[1][big]) <= 1.0001 * cap + 10).all()


@pytest.mark.parametrize("scale,cap", [(1.0, 1e-30), (1e10, 1e-30), (1e-30, 1e-28), (1e-20, 1.0), (1e-6, 1e30)])
@pytest.mark.parametrize("nq", [1, 12, 90])
def test_scales_and_caps_far_from_one(scale, cap, nq):
    p = Problem(nq + 1, ref.FP4, [[64, 64, 40]], [nq], 4, 2, 64)
    p.scale = float(np.float32(scale))
    cap = float(np.float32(cap))
    p.q[0] = 0.0                                             # scores of zero stay zero
    for masks in (dict(), dict(causal=True)):
        out, lse, mag, err = model(p, cap, **masks)
        # the raw score's error, which the formula bounds by its size, can move a score by twice the cap at most
        ref.check_attend(f"{masks}", *p.gpu(cap=cap, **masks), out, lse, mag, np.minimum(err, 2 * cap + 2.0 ** -19))
