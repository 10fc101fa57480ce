"""Keys and values that are no numbers, and places that hold whatever bytes."""
import numpy as np
import pytest
import torch

import kv_reference as ref
from test_gpu_kv import FMTS, Problem

pytestmark = pytest.mark.gpu

NQ = [1, 12, 90]     # tokens of four heads in two groups: tiles of 16, 32 and 128 rows


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("masks", [dict(causal=True), dict(causal=True, window=30), dict(causal=True, cap=5.0),
                                   dict(causal=True, bias=True)])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("name,d", [("bf16", 64), ("fp8", 64), ("fp8", 128), ("fp8", 256), ("fp4", 64), ("fp4", 128),
                                    ("fp4", 256)])
@pytest.mark.parametrize("nq", NQ)
def test_a_key_that_is_not_a_number_shows(name, d, nq, sign, masks):
    # NaN in the key alone; its block's codes say nothing, and queries of one sign add them up without cancelling
    fmt = FMTS[name]
    p = Problem(20 + d, fmt, [[64, 64, 64]], [nq], 4, 2, d)
    p.q = sign * p.q.abs()
    clean = p.model(**masks)
    at = 192 - nq // 2 - 2
    page, row, _ = p.ctx[0][at]
    codes, scales = ref.views(fmt, 32, 2, d, p.pool)[0]
    if fmt == ref.BF16:
        codes[page, :, row, 10:12] = (0xC0, 0x7F)
    else:
        scales[page, :, row, 1] = 255
        codes[page, :, row] = 0x11 if fmt == ref.FP4 else 0x30
    out, lse = p.gpu(**masks)
    qpos = np.arange(nq) + 192 - nq
    sees = (qpos >= at) & (qpos - masks.get("window", 1000) < at)
    if (~sees).any():
        ref.check_attend("rows that do not see it", *[x[~sees] for x in (out, lse, *clean)])
    assert np.isnan(out[sees]).all() and np.isnan(lse[sees]).all()


@pytest.mark.parametrize("tokens", [1, 31, 32, 64])
@pytest.mark.parametrize("masks", [dict(), dict(causal=True)])
@pytest.mark.parametrize("nq", NQ)
def test_a_value_shows_behind_keys_of_minus_infinity(nq, masks, tokens):
    # scores of -inf have weights of zero, and zero times such a value is no number: for one token as for whole units
    p = Problem(21, ref.BF16, [[64, 64, 64]], [nq], 4, 2, 64)
    p.q[..., 0] = 1.0
    page, row, _ = np.array(p.ctx[0][:tokens]).T
    keys, values = (v[0] for v in ref.views(ref.BF16, 32, 2, 64, p.pool))
    keys[page, :, row, 0:2] = (0x80, 0xFF)
    out, lse = p.gpu(**masks)
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    values[page, :, row, 10:12] = (0xC0, 0x7F)
    out, again = p.gpu(**masks)
    assert np.isnan(out[..., 5]).all() and np.array_equal(again, lse)


@pytest.mark.parametrize("name,d,byte", [("fp4", 64, 253), ("fp4", 128, 254), ("fp4", 256, 254), ("fp8", 64, 247),
                                         ("fp8", 128, 250), ("fp8", 256, 254), ("fp8", 256, 255)])
@pytest.mark.parametrize("nq", NQ)
def test_bytes_that_no_call_wrote_reach_nobody_who_does_not_see_them(name, d, byte, nq):
    # places within a chunk's length that hold something else: scales whose products leave the range of fp32
    fmt = FMTS[name]
    p = Problem(22 + d, fmt, [[64, 64, 64]], [nq], 4, 2, d)
    at = 160 if nq == 1 else 192 - nq // 2 - 2                   # (one token sees 162 to 191)
    masks = dict(causal=True, window=30)
    clean = p.model(**masks)
    page, row, _ = p.ctx[0][at]
    for codes, scales in ref.views(fmt, 32, 2, d, p.pool):
        codes[page, :, row] = 0x77 if fmt == ref.FP4 else 0x7E      # the largest values
        scales[page, :, row] = byte
    out, lse = p.gpu(**masks)
    qpos = np.arange(nq) + 192 - nq
    sees = (qpos >= at) & (qpos - 30 < at)
    assert (~sees).any()
    ref.check_attend("rows that do not see it", *[x[~sees] for x in (out, lse, *clean)])
