"""Keys that are stored as they come, and values, keep their bits: the sign of a zero, the payload of a NaN."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import DTYPES, ints

pytestmark = pytest.mark.gpu


def bits(x):
    return x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32).cpu()


def odd_values(rows, heads, D, dtype):
    """zeros of both signs, infinities, subnormals, and NaN with payloads and signs"""
    if dtype == torch.bfloat16:
        pool = torch.tensor([0x0000, -0x8000, 0x7f80, -0x0080, 0x0001, -0x7fff, 0x7fa5, 0x7fc1, -0x003f, 0x3f80], dtype=torch.int16)
    else:
        pool = torch.tensor([0, -2**31, 0x7f800000, -0x00800000, 1, -2**31 + 1, 0x7f812345, 0x7fc00001, -0x003fffff, 0x3f800000],
                            dtype=torch.int32)
    i = torch.arange(rows * heads * D) * 7 // 3 % pool.numel()
    return pool[i].view(dtype).view(rows, heads, D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [1, 7, 30, 36, 64, 72, 128, 256])
@pytest.mark.parametrize("heads", [1, 3, 8])
def test_keys_as_they_come(dtype, D, heads):
    rows, page = 9, 4
    k, v = odd_values(rows, heads, D, DTYPES[dtype]), odd_values(rows, heads, D, DTYPES[dtype]).flip(0).contiguous()
    kc, vc = (torch.zeros(4, page, heads, D, dtype=DTYPES[dtype], device="cuda") for _ in range(2))
    P.ttf_cache_append(k.cuda(), v.cuda(), kc, vc, ints([0, rows]), ints([rows]), ints([[2, 0, 3]]))
    assert P.ttf_paged_status() == 0
    for i in range(rows):
        g = [2, 0, 3][i // page]
        assert torch.equal(bits(kc[g, i % page]), bits(k[i])) and torch.equal(bits(vc[g, i % page]), bits(v[i]))
