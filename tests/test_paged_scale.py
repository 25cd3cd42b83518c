"""The factor of the scores: what the kernels can form, and what is refused."""
import ctypes

import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import build as B
from tests.test_gpu_attend import Batch
from tests.test_paged_refusals import INVALID, cache, heads, ref, sequences


def test_a_scale_that_no_power_of_two_holds():
    """scale log2(e) beyond the largest number: every score would be infinite or no number"""
    B.build()
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert P.lib().ttf_attend(ref(heads(8)), ref(sequences()), ref(cache()), ctypes.c_float(scale), 1, 0, ref(heads(8)), None) == INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 100])
def test_the_largest_scale(dtype, new):
    """scores of zero stay scores of zero: the mean of the values that a row sees"""
    b = Batch([new], [40], 16, 4, 2, 64, dtype, spare=0)
    b.q.zero_()
    b.scale = 2.3e38
    out = b.check()
    assert torch.isfinite(out).all()
