"""The count of ttf_rotate is one value: an array of none is not "all rows", and of several it is not clear which."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("outputs", [False, True])
def test_count_is_one_value(outputs):
    x, pos, freq = torch.ones(4, 2, 8, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda")
    out = dict(out_q=torch.zeros_like(x)) if outputs else {}
    for bad in (torch.empty(0, dtype=torch.int32, device="cuda"), ints([1, 2]), torch.empty((0, 3), dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            P.ttf_rotate(x, None, pos, freq, count=bad, **out)
    if outputs:
        assert (out["out_q"] == 0).all()
    for good in (ints([2]), ints(2), ints([[2]])):
        got = P.ttf_rotate(x, None, pos, freq, count=good, out_q=torch.zeros_like(x))[0]
        assert (got[2:] == 0).all() and (got[:2].abs().sum(-1) > 0).all()
