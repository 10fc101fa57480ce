"""Results and workspaces of calls on another stream than the current one."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2607_05708_amd as pm
from test_gpu_kv import Problem, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def allocations(monkeypatch, call):
    """(result, [(stream that a tensor was allocated on, its address, its bytes)]) of a call."""
    seen = []

    def spy(real):
        def f(*args, **kw):
            t = real(*args, **kw)
            seen.append((torch.cuda.current_stream().cuda_stream, t.data_ptr(), t.nbytes))
            return t
        return f

    with monkeypatch.context() as mp:
        for name in ("empty", "empty_like"):
            mp.setattr(torch, name, spy(getattr(torch, name)))
        return call(), seen


def test_calls_on_another_stream_take_that_streams_memory(monkeypatch):
    p = Problem(31, ref.FP8, [[64] * 12, [64, 5]], [3, 3], 4, 2, 128)
    cache, q, off, tok, ids = p.cache(), p.q.cuda(), up(p.off), up(p.tok_len), up(p.ids)
    chunk, pos = up(np.zeros(40, np.int32)), up(np.arange(40, dtype=np.int32))
    calls = [(2, lambda s: pm.mem_kv_read(cache, chunk, pos, stream=s)),
             (3, lambda s: pm.mem_attend(cache, tok, ids, q, p.scale, q_offsets=off, causal=True, stream=s))]
    side = torch.cuda.Stream()
    for count, call in calls:
        want, here = allocations(monkeypatch, lambda: call(None))
        assert [s for s, _, _ in here] == [torch.cuda.current_stream().cuda_stream] * count
        want = [t.clone() for t in want]
        torch.cuda.synchronize()
        # free memory of the current stream that would fit: some work there may still use it
        freed = [torch.empty(n, dtype=torch.uint8, device="cuda") for _, _, n in here]
        spans = [(t.data_ptr(), t.data_ptr() + t.nbytes) for t in freed]
        del freed
        got, there = allocations(monkeypatch, lambda: call(side))
        assert [s for s, _, _ in there] == [side.cuda_stream] * count
        for _, at, n in there:
            assert all(at >= b or at + n <= a for a, b in spans)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        same, there = allocations(monkeypatch, lambda: call(torch.cuda.current_stream()))
        assert [s for s, _, _ in there] == [torch.cuda.current_stream().cuda_stream] * count
        assert all(torch.equal(a, b) for a, b in zip(same, want))


def test_results_may_be_used_and_freed_on_the_current_stream():
    p = Problem(32, ref.FP4, [[64] * 12], [40], 4, 2, 128)
    cache, q, off, tok, ids = p.cache(), p.q.cuda(), up(p.off), up(p.tok_len), up(p.ids)
    want = pm.mem_attend(cache, tok, ids, q, p.scale, q_offsets=off)[0].float()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    sums = []
    for _ in range(20):                                      # a result is read here while the next call writes there
        out, _ = pm.mem_attend(cache, tok, ids, q, p.scale, q_offsets=off, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        sums.append(out.float())
        del out
    torch.cuda.synchronize()
    assert all(torch.equal(s, want) for s in sums)
