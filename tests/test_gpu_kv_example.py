"""The example of a turn over its memory, against the 64-bit model."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("n", [1, 37])
def test_a_turn_over_its_memory(n):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("attend_memory", os.path.join(ROOT, "examples", "attend_memory.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    g = torch.Generator("cuda").manual_seed(n)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    h, hq, d, m = ex.HEADS, ex.HEADS_Q, ex.HEAD_DIM, 2
    mem = ex.Memory(64)
    emb = rand(12, ex.EMB)
    past = mem.open(emb)
    mem.store(past, rand(12 * 45, h, d), rand(12 * 45, h, d))
    q, k, v = rand(m * n, hq, d), rand(m * n, h, d), rand(m * n, h, d)
    want = rand(m, ex.EMB)
    out, lse, ids = ex.turn(mem, want, q, k, v, 3)
    torch.cuda.synchronize()
    host = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    scores = host(want) @ host(emb).T
    pool, table, tok = mem.cache.pool.cpu().numpy(), mem.cache.table.cpu().numpy(), mem.tok_len.cpu().numpy()
    own = ref.encode_rows(ref.FP4, host(k))
    for i in range(m):
        best = np.sort(np.argsort(-scores[i])[:3])
        assert ids[i].tolist() == best.tolist() + [12 + i]
        pos = [(c, t) for c in ids[i].tolist() for t in range(tok[c])]
        assert len(pos) == 3 * 45 + n
        page, row = (np.array(x) for x in zip(*[(table[c, t // ex.PAGE_TOKENS], t % ex.PAGE_TOKENS) for c, t in pos]))
        kk, vv = ref.get(ref.FP4, ex.PAGE_TOKENS, h, d, pool, page, row)
        mine = [a[i * n:(i + 1) * n] for a in own]
        assert np.array_equal(kk[-n:], ref.decode_rows(ref.FP4, *mine))
        qpos = np.arange(n) + len(pos) - n
        expect = ref.attend(host(q)[i * n:(i + 1) * n], kk, vv, None, np.ones(len(pos), bool), qpos, None,
                            float(np.float32(1 / math.sqrt(d))), True, 0, 0, 0.0, None)
        ref.check_attend(f"request {i}", host(out)[i * n:(i + 1) * n], host(lse)[i * n:(i + 1) * n], *expect)
