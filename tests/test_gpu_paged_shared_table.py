"""A table whose rows are one and the same (a stride of zero): sequences that share all their pages."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import ints
from tests.test_gpu_attend import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 70, 9]])
def test_sequences_over_the_same_pages(dtype, new):
    b = Batch(new, [max(new) + 90 - n for n in new], 16, 4, 2, 64, dtype)
    q, k, v, st, ln, tb = b.on_device()
    shared = tb[:1].expand(3, -1)
    assert shared.stride(0) == 0
    want = P.ttf_attend(q, k, v, st, ln, shared.contiguous(), b.scale, out=torch.zeros_like(q))
    got = P.ttf_attend(q, k, v, st, ln, shared, b.scale, out=torch.zeros_like(q))
    assert P.ttf_paged_status() == 0 and torch.equal(got, want)


def test_append_of_rows_that_follow_one_another():
    """two sequences of one page list: the second one's token lies behind the first one's"""
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(4, 2, 32, generator=g).cuda() for _ in range(2))
    kc, vc = (torch.zeros(3, 4, 2, 32, device="cuda") for _ in range(2))
    P.ttf_cache_append(k, v, kc, vc, ints([0, 3, 4]), ints([3, 5]), ints([[2, 1]]).expand(2, -1))
    assert P.ttf_paged_status() == 0
    assert torch.equal(kc[2, :3], k[:3]) and torch.equal(kc[1, 0], k[3]) and torch.equal(vc[2, :3], v[:3]) and torch.equal(vc[1, 0], v[3])
    assert (kc[2, 3] == 0).all() and (kc[0] == 0).all()
