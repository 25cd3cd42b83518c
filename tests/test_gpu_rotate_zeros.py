"""Channels that do not turn, behind those that do, keep the sign of a zero."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import DTYPES, ints
from tests.test_gpu_append_bits import bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot", [(64, 32), (72, 36), (128, 64), (128, 0), (256, 128), (33, 10), (7, 4), (256, 250)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_channels_that_do_not_turn_keep_the_sign_of_zero(dtype, D, rot, interleaved):
    g = torch.Generator().manual_seed(D + rot)
    x = torch.randn(6, 3, D, generator=g).to(DTYPES[dtype])
    x[..., rot:] = torch.where(torch.rand(6, 3, D - rot, generator=g) < 0.5, 0.0, -0.0).to(x.dtype)
    pos, freq = torch.arange(6, dtype=torch.int32, device="cuda"), torch.rand(rot // 2, generator=g).cuda()
    got, _ = P.ttf_rotate(x.cuda(), None, pos, freq, rot_dim=rot, interleaved=interleaved)
    assert torch.equal(bits(got[..., rot:]), bits(x[..., rot:]))
    kc, vc = (torch.ones(2, 4, 3, D, dtype=x.dtype, device="cuda") for _ in range(2))
    P.ttf_cache_append(x.cuda(), x.cuda(), kc, vc, ints([0, 6]), ints([6]), ints([[1, 0]]), pos, freq, rot_dim=rot, interleaved=interleaved)
    assert torch.equal(bits(kc.flip(0).flatten(0, 1)[:6, :, rot:]), bits(x[..., rot:]))
