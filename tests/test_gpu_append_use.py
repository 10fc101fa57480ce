"""Keys and queries rotated on their way, then attended: against the 64-bit model of the rotation and of the attention."""
import numpy as np
import pytest
import torch

import kv_reference as kv
import latent_reference as ref
import paper_2607_05708_amd as pm
from test_gpu_append import FMTS, freqs, host, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("name", FMTS)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("shift,dim", [(0, 64), (1000, 64), (-70, 48), (500000, 16)])
def test_rotated_keys_and_queries_attended(name, pairs, shift, dim):
    fmt, n, heads, hq, d, T = FMTS[name], 60, 2, 6, 64, 32
    rng = np.random.default_rng(dim + shift % 97)
    rows = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(torch.bfloat16)  # noqa: E731
    k, v, q, f = rows(n, heads, d), rows(n, heads, d), 2 * rows(n, hq, d), freqs(dim)
    at = shift + np.arange(n)
    pool = torch.zeros((2, kv.page_bytes(fmt, T, heads, d)), dtype=torch.uint8, device="cuda")
    cache = pm.KvCache(pool, up(np.array([[1, 0]], np.int32)), T, heads, d, fmt)
    turned = pm.mem_kv_append(cache, k.cuda(), v.cuda(), up(np.zeros(n, np.int32)), up(np.arange(n, dtype=np.int32)),
                              up(at.astype(np.int32)), up(f), q=q.cuda(), pairs=pairs)
    got, lse = pm.mem_attend(cache, up(np.array([n], np.int32)), up(np.zeros((1, 1), np.int32)), turned, 0.125,
                             causal=True)
    k, v, q = (x.double().numpy() for x in (k, v, q))
    rest = (None, np.ones(n, bool), np.arange(n), None, 0.125, True, 0, 0, 0.0, None)

    def model(kk, qq):
        held = [kv.decode_rows(fmt, *kv.encode_rows(fmt, x)) for x in (kk, v)]
        return kv.attend(kv.to_bf16(qq), *held, *rest)

    got, lse = host(got), host(lse)
    kv.check_attend("rotated", got, lse, *model(ref.rotate(k, at, f, pairs), ref.rotate(q, at, f, pairs)))
    for wrong in (model(k, q), model(ref.rotate(k, at, f, pairs), q), model(k, ref.rotate(q, at, f, pairs)),
                  model(ref.rotate(k, at, f, not pairs), ref.rotate(q, at, f, not pairs))):
        with pytest.raises(AssertionError):
            kv.check_attend("without it, or with the other pairs", got, lse, *wrong)
