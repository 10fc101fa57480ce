"""Latent attention with exact scores, so that tolerances are close: one rounding too many or a lost unit of the context
shows.  Contexts of so many units that workgroups resolve them in several batches; the choice of the form."""
import numpy as np
import pytest
import torch

import latent_reference as ref
import paper_2607_05708_amd as pm
from latent_exact import ABSORBED, EXPANDED, Exact
from test_gpu_latent import FMTS, FORMS, Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# heads and new tokens a request: tiles of 16, 64 and 128 rows in the absorbed form
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("h,nq", [(3, 1), (40, 1), (16, 9)])
@pytest.mark.parametrize("name,latent,d", [("fp4", 512, 128), ("fp8", 256, 64), ("fp8", 512, 64), ("bf16", 256, 128),
                                           ("bf16", 512, 128)])
@pytest.mark.parametrize("even", [True, False])
def test_outputs_are_rounded_as_documented(form, h, nq, name, latent, d, even):
    lens = [[3], [40], [64, 33], [64] * 5, [1], [12, 64]]
    p = Exact(h + latent + d, FMTS[name], lens, [nq] * len(lens), h, d, latent, even=even)
    out, lse = p.gpu(form)
    sample = [(j // nq, j, x) for j in range(len(p.q)) for x in range(0, h, 1 + h // 4)]
    print("worst", p.check_rows(form, sample, out, lse))


def one_part_bytes(p, form, k):
    """Workspace of a call whose contexts are not split: rows, heads and units as the header's forms need them."""
    up256 = lambda b: (b + 255) // 256 * 256  # noqa: E731
    rows, m, units = len(p.q) * p.h, len(p.nq), k * p.table.shape[1] * p.T // 32
    if form == ABSORBED:
        return up256(rows * (p.latent + 64) * 2) + up256(rows * p.latent * 4) + up256(rows * 8)
    slots = m * units * 32
    heads = min(max((1 << 30) // (slots * (2 * p.d + 64) * 2), 1), p.h)
    return (up256(m * units * 16) + up256(2 * m * 4) + up256(heads * slots * (p.d + 64) * 2)
            + up256(heads * slots * p.d * 2))


BATCHES = [  # form, format, elements, heads of, requests, new tokens, heads: units resolved at a time
    (ABSORBED, "fp8", 512, 128, 256, 1, 16, 128), (ABSORBED, "bf16", 512, 64, 256, 1, 5, 128),
    (ABSORBED, "fp4", 256, 64, 512, 1, 16, 128), (ABSORBED, "fp4", 512, 128, 256, 1, 40, 64),
    (ABSORBED, "bf16", 256, 64, 256, 1, 64, 64), (ABSORBED, "fp8", 512, 128, 256, 1, 128, 64),
    (ABSORBED, "bf16", 512, 128, 64, 32, 16, 64), (ABSORBED, "fp4", 512, 64, 64, 32, 16, 64),
    (ABSORBED, "fp8", 256, 64, 64, 32, 16, 64), (EXPANDED, "fp8", 512, 128, 8, 512, 16, 128),
    (EXPANDED, "bf16", 256, 64, 8, 512, 16, 128)]


@pytest.mark.parametrize("form,name,latent,d,m,nq,h,batch", BATCHES)
def test_contexts_of_several_batches_of_units(form, name, latent, d, m, nq, h, batch):
    # every request reads one context of 5,400 tokens, some of whose first units are not full, through a window that ends
    # among its first 140 tokens, where a value is not finite: it reaches the rows that see it and no other
    rng = np.random.default_rng(latent + m + h)
    lens = [64, 5, 33, 64, 1] + [64] * 30 + [47] + [64] * 50
    n, at = sum(lens), 70
    p = Exact(latent + h, FMTS[name], [lens] + [[]] * (m - 1), [nq] * m, h, d, latent)
    p.ids[:] = p.ids[0]
    p.ctx = [p.ctx[0]] * m
    masks = dict(causal=True, window=n - 140)
    q_pos = n - 1 - rng.integers(0, 140, m * nq)
    cache = p.cache()
    need = pm.mem_latent_attend_workspace_bytes(cache, m, len(lens), m * nq, h, d, form)
    assert need == one_part_bytes(p, form, len(lens)), "contexts are split: a workgroup has fewer units"
    assert (n - 280) // 32 > batch, "the units of one batch"
    page, row, _ = p.ctx[0][at]
    for value in (None, np.nan):
        if value is not None:
            c, r = ref.get(p.fmt, p.T, latent, p.pool, page, row)
            c[133] = value
            ref.put(p.fmt, p.T, p.pool, page, row, c, r)
        out, lse = p.gpu(form, q_pos=q_pos, offsets=False, **masks)
        touched = (q_pos - masks["window"] < at) & (value is not None)
        finite = np.isfinite(out).all((1, 2))
        assert np.array_equal(finite, ~touched)
        assert not np.isfinite(out[touched]).any()
        rows = rng.permutation(np.flatnonzero(~touched))[:10]
        sample = [(j // nq, j, int(x)) for j in rows for x in rng.permutation(h)[:2]]
        print("worst", p.check_rows(form, sample, out, lse, q_pos=q_pos, **masks))


@pytest.mark.parametrize("latent,d,at", [(512, 128, 171), (256, 64, 86)])
def test_the_form_that_is_chosen(latent, d, at):
    # new tokens a request, rounded down: d latent / (latent - d) is passed at `at`
    for m, nq in ((1, at - 1), (1, at), (3, at - 1), (3, at)):
        p = Problem(nq + m, FMTS["fp8"], [[64, 64, 64, 64, 9]] * m, [nq] * m, 2, d, latent)
        form = EXPANDED if nq == at else ABSORBED
        cache, k = p.cache(), p.ids.shape[1]
        sizes = [pm.mem_latent_attend_workspace_bytes(cache, m, k, m * nq, 2, d, f) for f in (0, form, 3 - form)]
        assert sizes[0] == sizes[1] != sizes[2]
        space = torch.empty(sizes[0], dtype=torch.uint8, device="cuda")
        got, want, other = (p.gpu(f, cache=cache, causal=True, workspace=w)
                            for f, w in ((0, space), (form, space), (3 - form, None)))
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
        assert not np.array_equal(got[0], other[0])

