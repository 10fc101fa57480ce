"""Which sizes the latent calls take, without a GPU: the check of a call's launches comes before that of its workspace,
so that a call without one says which of the two it fails."""
import ctypes as C
import os

import pytest

import paper_2607_05708_amd as pm
from test_latent_abi import FAKE, FAR, _latent, _p, _rows

pytestmark = pytest.mark.skipif(not os.path.exists(pm.library_path()), reason="libmemattn.so not built")
UNSUPPORTED, WORKSPACE = -2, -3
ABSORBED, EXPANDED = 1, 2


def status(m, k, total_q, heads, form, q_offsets=None, **cache):
    """Of mem_latent_attend without a workspace: 512 elements, heads of 128."""
    a = pm.MemAttendArgs(FAKE, FAKE, m, k, heads, q_offsets, None, 0.1, 0.0, None, 0, 0, None, None, None)
    w = pm.MemLatentWeights(FAKE, 256 * 512, 512, 128)
    return pm.lib().mem_latent_attend(_p(_latent(**cache)), C.byref(a), _p(_rows()), _p(_rows(2 * FAR)), total_q,
                                      C.byref(w), form, FAKE, None, None, 0, None)


@pytest.mark.parametrize("ragged", [None, FAKE])
@pytest.mark.parametrize("m,k,heads", [(64, 512, 128), (64, 4096, 16), (16, 2048, 128), (256, 1024, 1024)])
def test_expanded_form_takes_large_capacities_of_many_heads(m, k, heads, ragged):
    # chunks of 512 tokens: 4 m k workgroups make keys and values, whatever the number of heads
    groups = m * k * 512 // 32 // 4
    assert groups < (1 << 24) - 1 <= groups * heads
    for form in (EXPANDED, 0):
        assert status(m, k, m * 256, heads, form, ragged) == WORKSPACE, (form, pm.lib().mem_last_error())


@pytest.mark.parametrize("m,k,page_tokens,ppc", [(1 << 22, 16, 64, 8), (4096, 4096, 64, 8)])
def test_more_groups_of_units_than_a_launch_has_are_refused(m, k, page_tokens, ppc):
    assert m * k * page_tokens * ppc // 32 // 4 > (1 << 24) - 1
    for heads in (1, 2):
        assert status(m, k, m, heads, EXPANDED, page_tokens=page_tokens, ppc=ppc) == UNSUPPORTED


def test_the_new_tokens_of_an_absorbed_call():
    # 65,535 groups of 32 tokens each
    most = 65535 * 32
    assert status(most, 1, most, 16, ABSORBED) == WORKSPACE
    assert status(most + 1, 1, most + 1, 16, ABSORBED) == UNSUPPORTED


@pytest.mark.parametrize("m,total_q,form", [(1, 512, EXPANDED), (1, 170, ABSORBED), (4, 684, EXPANDED),
                                            (4, 683, ABSORBED), (64, 16384 + 63, EXPANDED)])
def test_the_form_goes_by_the_mean_of_the_new_tokens(m, total_q, form):
    # 512 elements, heads of 128: from 171 new tokens a request on, whichever request has them and whatever they see
    size = lambda f: pm.lib().mem_latent_attend_workspace_bytes(C.byref(_latent()), m, 48, total_q, 16, 128, f)  # noqa: E731
    assert size(0) == size(form) != size(3 - form)


def test_the_memory_of_the_expanded_form():
    # keys and values of the whole capacity, of one head at least: m k page_tokens pages_per_chunk (2 head_dim + 64) 2 bytes
    size = lambda m, k, form: pm.lib().mem_latent_attend_workspace_bytes(C.byref(_latent()), m, k, m * 256, 16, 128,  # noqa: E731
                                                                         form)
    one_head = 64 * 4096 * 512 * 320 * 2
    assert one_head < size(64, 4096, EXPANDED) < 1.03 * one_head        # (and 1 / 2 byte a token of where its units lie)
    assert size(64, 4096, 0) == size(64, 4096, EXPANDED) > 10 * size(64, 4096, ABSORBED)
    assert size(64, 64, EXPANDED) < 1.1 * 2 ** 30 + 64 * 64 * 512 * 640  # else as many heads as 1 GiB holds
