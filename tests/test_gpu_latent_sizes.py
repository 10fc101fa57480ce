"""Latent attention at the ends of its sizes, against the 64-bit model."""
import pytest
import torch

import latent_reference as ref
import paper_2607_05708_amd as pm
from test_gpu_latent import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_many_heads_over_a_long_and_nearly_empty_list():
    # 16,384 groups of units of 1,024 heads each: 2^24 together
    p = Problem(5, pm.MEM_KV_FP4, [[512, 100, 3]], [2], 1024, 64, 256, page_tokens=64, ppc=8, k=4096, holes=True)
    p.check("many heads", forms=[ref.EXPANDED], causal=True)
