"""The model of exact scores: that its tolerances are close enough to show a lost half of a sum or of a weight, or a unit
of the context left out (mistakes made in the model)."""
import numpy as np
import pytest

import latent_exact as exact
import paper_2607_05708_amd as pm


@pytest.mark.parametrize("name,latent,d", [("fp8", 512, 128), ("bf16", 256, 64)])
@pytest.mark.parametrize("lens", [[3], [40], [64, 33]])
@pytest.mark.parametrize("mistake,even,rows", [("one_sum", True, 16), ("one_sum", True, 64), ("one_sum", True, 128),
                                               ("one_sum", False, 16), ("one_weight", False, 16)])
def test_one_rounding_too_many_shows(name, latent, d, lens, mistake, even, rows):
    fmt = {"fp8": pm.MEM_KV_FP8, "bf16": pm.MEM_KV_BF16}[name]
    p = exact.Exact(sum(lens), fmt, [lens], [4], 3, d, latent, even=even)
    c, r = p.tokens(0)
    see = np.ones(len(c), bool)
    wrong = 0
    for j in range(4):
        for x in range(3):
            want, _, tol, _ = p.row(exact.ABSORBED, rows, 0, j, x, see, c, r)
            got, _, _, _ = p.row(exact.ABSORBED, rows, 0, j, x, see, c, r, **{mistake: True})
            wrong += int((np.abs(got - want) > tol).sum())
    assert wrong >= 5, "a kernel that rounds once more would pass"


@pytest.mark.parametrize("form,rows", [(exact.ABSORBED, 16), (exact.ABSORBED, 64), (exact.ABSORBED, 128),
                                       (exact.EXPANDED, 128)])
def test_a_unit_left_out_shows(form, rows):
    p = exact.Exact(1, pm.MEM_KV_FP8, [[64] * 80], [1], 2, 128, 512)
    c, r = p.tokens(0)
    see = np.ones(len(c), bool)
    less = see.copy()
    less[1024:1056] = False
    for x in range(2):
        _, want, _, tol = p.row(form, rows, 0, 0, x, see, c, r)
        _, got, _, _ = p.row(form, rows, 0, 0, x, less, c, r)
        assert abs(got - want) > 4 * tol
