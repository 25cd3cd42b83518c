"""Contexts of so few blocks that the tcgen05 kernel's producer is through before anybody's wait runs out: the CTA stays until its
copies have landed, so that the CTA after it finds its shared memory to itself."""
import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import binding as B
from tests.test_gpu_attend import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,before", [([100], [28]), ([128], [0]), ([100, 120], [156, 136]), ([60], [1]), ([200], [2872])])
def test_waits_that_run_out_behind_the_producer(new, before, D):
    """one and two whole blocks, a part of a block, and eight CTAs that share the blocks"""
    b, c = Batch(new, before, 64, 8, 2, D), Batch([300, 70], [500, 90], 32, 8, 2, D, seed=5)
    mine, next_ = b.on_device(), c.on_device()
    want = P.ttf_attend(*mine, b.scale, out=torch.zeros_like(mine[0]))
    after = P.ttf_attend(*next_, c.scale, out=torch.zeros_like(next_[0]))
    assert P.ttf_paged_status() == B.TTF_OK
    for _ in range(10):
        P.ttf_debug_set_wait(32, 16)
        try:
            P.ttf_attend(*mine, b.scale, out=torch.zeros_like(mine[0]))
        finally:
            P.ttf_debug_set_wait()
        got = P.ttf_attend(*next_, c.scale, out=torch.zeros_like(next_[0]))      # the next CTAs on the same SMs
        assert P.ttf_paged_status() == B.TTF_ERR_TIMEOUT and torch.equal(got, after)
    assert torch.equal(P.ttf_attend(*mine, b.scale, out=torch.zeros_like(mine[0])), want) and P.ttf_paged_status() == B.TTF_OK
