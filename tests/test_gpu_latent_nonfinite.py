"""Latent attention over latent values and key parts that are not finite, in units that every row sees whole (no mask
clears or notes anything there) and behind scores of minus infinity."""
import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2607_05708_amd as pm
from test_gpu_latent import FMTS, FORMS, Problem, host

pytestmark = pytest.mark.gpu

# heads and new tokens a request: tiles of 16, 64 and 128 rows in the absorbed form
TILES = [(3, 1), (40, 1), (16, 9)]


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def set_latent(p, req, tokens, element, value):
    """Element of some tokens' latent vectors; "code": the 8-bit code of a NaN, its block's scale as it is."""
    for i in tokens:
        page, row, _ = p.ctx[req][i]
        if value == "code":
            codes, _, _ = ref.views(p.fmt, p.T, p.latent, p.pool)
            codes[page, row, element] = 0x7F
            continue
        c, r = ref.get(p.fmt, p.T, p.latent, p.pool, page, row)
        c[element] = value
        ref.put(p.fmt, p.T, p.pool, page, row, c, r)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("h,nq", TILES)
@pytest.mark.parametrize("latent,d", [(256, 64), (512, 128)])
@pytest.mark.parametrize("name,value", [("bf16", np.nan), ("bf16", np.inf), ("bf16", -np.inf), ("fp8", np.nan),
                                        ("fp8", "code"), ("fp4", np.nan)])
def test_in_a_unit_that_every_row_sees(form, h, nq, latent, d, name, value):
    p = Problem(7 * h + latent, FMTS[name], [[64, 64, 64], [64, 32]], [nq, nq], h, d, latent)
    other = [x[nq:] for x in p.model(form)]
    set_latent(p, 0, [70], 133, value)
    out, lse = p.gpu(form)
    finite = int(np.isfinite(out[:nq]).sum())
    assert finite == 0
    ref.check_attend("the other request", out[nq:], lse[nq:], *other)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("h,nq", TILES)
@pytest.mark.parametrize("latent,d", [(256, 64), (512, 128)])
def test_infinite_values_of_all_tokens_behind_scores_of_minus_infinity(form, h, nq, latent, d):
    # whichever of the infinities makes a row's scores: plus (no number is left of its softmax) or minus (no weight is)
    p = Problem(9 * h + latent, FMTS["bf16"], [[64, 32], [64]], [nq, nq], h, d, latent)
    other = [x[nq:] for x in p.model(form)]
    set_latent(p, 0, range(96), 133, np.inf)
    out, lse = p.gpu(form)
    finite = int(np.isfinite(out[:nq]).sum())
    assert finite == 0
    ref.check_attend("the other request", out[nq:], lse[nq:], *other)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("h,nq", TILES)
def test_infinite_key_parts_of_all_tokens_leave_nothing(form, h, nq):
    # scores of minus infinity weigh nothing: all finite values, so zeros as if nothing were seen
    p = Problem(11 * h, FMTS["fp8"], [[64, 32]], [nq], h, 64, 256)
    _, parts, _ = ref.views(p.fmt, p.T, p.latent, p.pool)
    for page, row, _ in p.ctx[0]:
        parts[page, row, 10:12] = (0x80, 0x7F)
    out, lse = p.gpu(form)
    below = host(p.t)[:, :, 5] < 0
    assert below.any() and not below.all()
    assert (out[below] == 0).all() and np.isneginf(lse[below]).all()
    finite = int(np.isfinite(out[~below]).sum())
    assert finite == 0


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("h,nq", TILES)
def test_infinite_values_of_all_tokens_of_a_split_context(form, h, nq):
    # full units alone: 240 of them, so that several workgroups have a part each
    p = Problem(13 * h, FMTS["bf16"], [[64] * 120], [nq], h, 64, 256)
    codes, _, _ = ref.views(p.fmt, p.T, p.latent, p.pool)
    codes[:, :, 2 * 133:2 * 133 + 2] = (0x80, 0x7F)
    out, lse = p.gpu(form)
    finite = int(np.isfinite(out).sum())
    assert finite == 0
