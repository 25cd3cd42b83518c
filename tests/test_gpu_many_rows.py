"""As many rows as an int counts: the loop over rows ends where they end."""
import ctypes

import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200.binding import TTFHeads, TTFRotation

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [2**31 - 1, 2**31 - 2961, 2**31 - 2960])
def test_a_norm_of_all_rows_an_int_can_count(rows):
    """one head of one channel, in place: y = x w / |x| = +-w, and what lies behind the rows is left alone"""
    x = torch.full((rows + 5,), -3.0, dtype=torch.bfloat16, device="cuda")
    weight = torch.full((1,), 2.0, dtype=torch.bfloat16, device="cuda")
    h = TTFHeads(x.data_ptr(), 1, 1, 1)
    turn = TTFRotation(freq=None, rot_dim=0, interleaved=0, axes=1, section=(0, 0, 0), cyclic=0, factor=1.0, q_weight=weight.data_ptr(),
                       k_weight=None, eps=0.0)
    ref = ctypes.byref
    assert P.lib().ttf_rotate(ref(h), None, 1, P.TTF_DTYPE_BF16, rows, None, None, ref(turn), ref(h), None, None) == 0
    torch.cuda.synchronize()
    assert P.ttf_paged_status() == 0
    assert (x[rows:] == -3).all()
    for at in range(0, rows, 1 << 28):
        assert (x[at:min(rows, at + (1 << 28))] == -2).all(), at
