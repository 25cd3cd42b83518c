"""What ttf_rotate, ttf_cache_append, ttf_attend and ttf_paged_status refuse, before any CUDA call: at the C ABI with
addresses that are never followed, and in the binding."""
import ctypes

import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import build as B
from paper_2605_07355_b200.binding import TTFCache, TTFHeads, TTFRotation, TTFSequences

INVALID, UNSUPPORTED = 1, 2


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.lib()


def heads(n=4, data=4096, row=512, head=128):
    return TTFHeads(data, row, head, n)


def rotation(**kw):
    r = TTFRotation(freq=4096, rot_dim=128, interleaved=0, axes=3, section=(24, 20, 20), cyclic=1, factor=1.0, q_weight=None,
                    k_weight=None, eps=1e-6)
    for k, v in kw.items():
        setattr(r, k, (ctypes.c_int * 3)(*v) if k == "section" else v)
    return r


def cache(**kw):
    c = TTFCache(k=4096, v=8192, k_page=16 * 512, k_row=512, k_head=128, v_page=16 * 512, v_row=512, v_head=128, pages=8,
                 page_size=16, heads=4, head_dim=128, dtype=1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def sequences(**kw):
    s = TTFSequences(start=4096, length=4096, table=4096, table_stride=4, table_pages=4, seqs=2, rows=10)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_rotate(lib):
    def call(q=heads(), k=heads(), dim=128, dtype=1, rows=10, pos=4096, rot=rotation(), oq=heads(), ok=heads()):
        return lib.ttf_rotate(ref(q), ref(k), dim, dtype, rows, None, pos, ref(rot), ref(oq), ref(ok), None)

    assert call(q=None, k=None, oq=None, ok=None) == INVALID
    assert call(oq=None) == INVALID and call(k=None) == INVALID
    assert call(q=heads(data=None)) == INVALID and call(ok=heads(data=None)) == INVALID
    assert call(q=heads(0), oq=heads(0)) == INVALID and call(q=heads(3)) == INVALID and call(ok=heads(5)) == INVALID
    assert call(dim=0) == INVALID and call(dtype=2) == INVALID and call(rows=0) == INVALID and call(rows=-1) == INVALID
    assert call(dim=257) == UNSUPPORTED
    assert call(pos=None) == INVALID and call(rot=None) == INVALID
    assert call(q=heads(65536), oq=heads(65536)) == UNSUPPORTED
    assert call(rows=2**30) == UNSUPPORTED                                                 # rows * heads
    assert call(q=heads(row=2**60), rows=100) == UNSUPPORTED
    for bad in (dict(rot_dim=-2), dict(rot_dim=3), dict(rot_dim=130), dict(axes=0), dict(axes=4), dict(interleaved=2),
                dict(cyclic=-1), dict(factor=float("nan")), dict(factor=float("inf")), dict(eps=-1.0), dict(eps=float("nan")),
                dict(freq=None), dict(section=(24, 20, 19)), dict(section=(84, -10, -10)), dict(section=(20, 22, 22)),
                dict(section=(0, 0, 64)), dict(section=(2**31 - 1, 2**31 - 1, 66), cyclic=0)):
        assert call(rot=rotation(**bad)) == INVALID, bad


def test_cache_append(lib):
    def call(k=heads(), v=heads(), q=heads(8), pos=4096, rot=rotation(), seq=sequences(), c=cache(), oq=heads(8)):
        return lib.ttf_cache_append(ref(k), ref(v), ref(q), pos, ref(rot), ref(seq), ref(c), ref(oq), None)

    assert call(k=None) == INVALID and call(v=None) == INVALID and call(oq=None) == INVALID and call(q=None) == INVALID
    assert call(rot=None) == INVALID                                                       # queries need a rotation
    assert call(k=heads(3)) == INVALID and call(v=heads(5)) == INVALID and call(q=heads(7)) == INVALID
    assert call(pos=None) == INVALID and call(seq=None) == INVALID and call(c=None) == INVALID
    check_cache_and_sequences(call)


def test_attend(lib):
    def call(q=heads(8), seq=sequences(), c=cache(), scale=0.1, causal=1, window=0, out=heads(8)):
        return lib.ttf_attend(ref(q), ref(seq), ref(c), scale, causal, window, ref(out), None)

    assert call(q=None) == INVALID and call(out=None) == INVALID and call(seq=None) == INVALID and call(c=None) == INVALID
    assert call(q=heads(7), out=heads(7)) == INVALID and call(q=heads(8), out=heads(4)) == INVALID
    assert call(q=heads(2), out=heads(2)) == INVALID                                       # fewer than the cache has
    assert call(scale=float("nan")) == INVALID and call(scale=float("inf")) == INVALID
    assert call(causal=2) == INVALID and call(causal=-1) == INVALID and call(window=-1) == INVALID
    check_cache_and_sequences(call)


def check_cache_and_sequences(call):
    for bad in (dict(k=None), dict(v=None), dict(pages=0), dict(page_size=0), dict(page_size=-1), dict(heads=0), dict(head_dim=0),
                dict(dtype=2), dict(dtype=-1)):
        assert call(c=cache(**bad)) == INVALID, bad
    assert call(c=cache(head_dim=257)) == UNSUPPORTED
    assert call(c=cache(k_page=2**61)) == UNSUPPORTED
    for bad in (dict(start=None), dict(length=None), dict(table=None), dict(table_stride=3), dict(table_pages=0), dict(seqs=0),
                dict(rows=0), dict(rows=-5)):
        assert call(seq=sequences(**bad)) == INVALID, bad


def test_status(lib):
    assert lib.ttf_paged_status(None, None) == INVALID


def test_structs_are_those_of_the_header():
    """sizes by the C rules: the binding's ctypes structs are what the marshalling and C programs pass"""
    assert ctypes.sizeof(TTFHeads) == 32 and ctypes.sizeof(TTFSequences) == 48
    assert ctypes.sizeof(TTFCache) == 88 and ctypes.sizeof(TTFRotation) == 64


def test_host_tensors_are_refused():
    x, i = torch.zeros(2, 4, 8), torch.zeros(2, dtype=torch.int32)
    c, t = torch.zeros(3, 4, 4, 8), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.ttf_rotate(x, None, i, torch.zeros(4))
    with pytest.raises(ValueError):
        P.ttf_rotate(None, None, i, torch.zeros(4))
    with pytest.raises(ValueError):
        P.ttf_cache_append(x, x, c, c, i, i[:1], t)
    with pytest.raises(ValueError):
        P.ttf_attend(x, c, c, i, i[:1], t, 1.0)


@pytest.mark.gpu
def test_the_binding_refuses_what_does_not_fit():
    dev = "cuda"
    x = torch.zeros(2, 4, 8, device=dev)
    k = torch.zeros(2, 2, 8, device=dev)
    pos, freq = torch.zeros(2, dtype=torch.int32, device=dev), torch.zeros(4, device=dev)
    start, length = (torch.tensor(v, dtype=torch.int32, device=dev) for v in ([0, 2], [2]))
    table, c = torch.zeros(1, 1, dtype=torch.int32, device=dev), torch.zeros(3, 4, 2, 8, device=dev)

    def refused(f, *a, **kw):
        with pytest.raises((ValueError, TypeError)):
            f(*a, **kw)

    P.ttf_rotate(x, k, pos, freq)
    refused(P.ttf_rotate, x.half(), None, pos, freq)
    refused(P.ttf_rotate, x, k.bfloat16(), pos, freq)
    refused(P.ttf_rotate, x, k[:1], pos, freq)
    refused(P.ttf_rotate, x, k[..., :6], pos, freq)
    refused(P.ttf_rotate, x.transpose(0, 2), None, pos, freq)
    refused(P.ttf_rotate, x, k, pos.long(), freq)
    refused(P.ttf_rotate, x, k, pos[:1], freq)
    refused(P.ttf_rotate, x, k, pos.cpu(), freq)
    refused(P.ttf_rotate, x, k, pos, freq.double())
    refused(P.ttf_rotate, x, k, pos, freq[:3])
    refused(P.ttf_rotate, x, k, pos.expand(3, 2).t(), freq, sections=(2, 1, 1))
    refused(P.ttf_rotate, x, k, pos.repeat(3, 1).t().contiguous(), freq)
    refused(P.ttf_rotate, x, k, pos, freq, sections=(2, 2))
    refused(P.ttf_rotate, x, k, pos, freq, q_weight=torch.zeros(8))
    refused(P.ttf_rotate, x, k, pos, freq, k_weight=torch.zeros(7, device=dev))
    refused(P.ttf_rotate, x, k, pos, freq, out_q=k)
    refused(P.ttf_rotate, x, None, pos, freq, out_k=k)
    refused(P.ttf_rotate, x, k, pos, freq, count=torch.zeros(1, device=dev))
    P.ttf_cache_append(k, k, c, c.clone(), start, length, table, pos, freq, q=x)
    refused(P.ttf_cache_append, k, k[:1], c, c, start, length, table)
    refused(P.ttf_cache_append, k, k, c, c[:2], start, length, table)
    refused(P.ttf_cache_append, k, k, c.bfloat16(), c.bfloat16(), start, length, table)
    refused(P.ttf_cache_append, k, k, c.transpose(1, 3), c.transpose(1, 3), start, length, table)
    refused(P.ttf_cache_append, k, k, c, c, start[:1], length, table)
    refused(P.ttf_cache_append, k, k, c, c, start, length.long(), table)
    refused(P.ttf_cache_append, k, k, c, c, start, length, table[0])
    refused(P.ttf_cache_append, k, k, c, c, start, length, table, pos)
    refused(P.ttf_cache_append, k, k, c, c, start, length, table, q=x)
    refused(P.ttf_cache_append, k, k, c, c, start, length, table, k_weight=freq)
    P.ttf_attend(x, c, c, start, length, table, 1.0)
    refused(P.ttf_attend, x, c[..., :6], c[..., :6], start, length, table, 1.0)
    refused(P.ttf_attend, x, c, c, start, length, table, 1.0, out=k)
    refused(P.ttf_attend, x, c, c, start, length, table.expand(1, 1).cpu(), 1.0)
    with pytest.raises(P.TTFError):
        P.ttf_attend(x[:, :3], c, c, start, length, table, 1.0)              # three query heads over two
    with pytest.raises(P.TTFError):
        P.ttf_attend(x, c, c, start, length, table, float("nan"))
    # no rows: nothing to do
    e = x[:0]
    assert P.ttf_rotate(e, None, pos[:0], freq)[0].shape == e.shape and P.ttf_attend(e, c, c, start, length, table, 1.0).shape == e.shape
