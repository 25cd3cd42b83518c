"""Strides of zero: inputs may have them (one head's memory for all heads, one page for every entry), outputs may not."""
import ctypes

import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import build as B
from tests.paged import attend_ref, rotate_ref, worst
from tests.test_gpu_attend import Batch
from tests.test_paged_refusals import INVALID, cache, heads, ref, rotation, sequences


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.lib()


def test_outputs_in_one_place_are_refused(lib):
    h, s, c, r = heads(), sequences(), cache(), rotation()
    for bad in (heads(head=0), heads(row=0)):
        assert lib.ttf_rotate(ref(h), None, 128, 1, 10, None, 4096, ref(r), ref(bad), None, None) == INVALID
        assert lib.ttf_rotate(None, ref(h), 128, 1, 10, None, 4096, ref(r), None, ref(bad), None) == INVALID
        assert lib.ttf_cache_append(ref(h), ref(h), ref(h), 4096, ref(r), ref(s), ref(c), ref(bad), None) == INVALID
        assert lib.ttf_attend(ref(h), ref(s), ref(c), ctypes.c_float(1.0), 1, 0, ref(bad), None) == INVALID
    for axis in ("k_page", "k_row", "k_head", "v_page", "v_row", "v_head"):
        bad = cache(**{axis: 0})
        assert lib.ttf_cache_append(ref(h), ref(h), None, 4096, ref(r), ref(s), ref(bad), None, None) == INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1], [3, 8], [100, 40]])
@pytest.mark.parametrize("what", ["q heads", "q rows", "cache heads", "cache rows", "cache pages"])
def test_attention_of_broadcast_inputs(dtype, new, what):
    b = Batch(new, [40, 200], 16, 8, 4, 64, dtype)
    q, k, v, st, ln, tb = b.on_device()
    if what == "q heads":
        b.q, q = b.q[:, :1].expand_as(b.q), q[:, :1].expand_as(q)
    elif what == "q rows":
        b.q, q = b.q[:1].expand_as(b.q), q[:1].expand_as(q)
    else:
        def cut(x):
            return {"cache heads": x[:, :, :1], "cache rows": x[:, :1], "cache pages": x[:1]}[what].expand_as(x)
        b.k, b.v, k, v = cut(b.k), cut(b.v), cut(k), cut(v)
    m = b.start[-1]
    out = P.ttf_attend(q, k, v, st, ln, tb, b.scale)
    assert out.stride() == (8 * 64, 64, 1) and P.ttf_paged_status() == 0
    want, tol = attend_ref(b.q, b.k, b.v, b.start, b.length, b.table, b.scale)
    assert worst(out[:m].cpu(), want[:m], tol[:m]) <= 1


@pytest.mark.gpu
def test_rotation_of_broadcast_heads():
    g = torch.Generator().manual_seed(3)
    x = torch.randn(9, 1, 64, generator=g).bfloat16().expand(9, 6, 64)
    pos, freq = torch.arange(9, dtype=torch.int32), torch.rand(32, generator=g)
    got, _ = P.ttf_rotate(x[:, :1].cuda().expand(9, 6, 64), None, pos.cuda(), freq.cuda())
    want, tol = rotate_ref(x, pos, freq)
    assert worst(got.cpu(), want, tol) <= 1
