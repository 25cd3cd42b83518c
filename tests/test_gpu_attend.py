"""ttf_attend against the definition in 64 bits (tests/paged.py)."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import DTYPES, attend_ref, ints, spread_pages, starts, worst

pytestmark = pytest.mark.gpu


class Batch:
    def __init__(self, new, before, page, heads, kv_heads, D, dtype="bf16", seed=0, spare=2, heads_first=False, pad=0, size=1.5):
        g = torch.Generator().manual_seed(seed + sum(new) + D)
        dt = DTYPES[dtype]
        self.new, self.length = new, [a + b for a, b in zip(new, before)]
        self.start, self.rows = starts(new), sum(new) + spare
        self.table, pages = spread_pages(self.length, page, g)
        wide = (size * torch.randn(self.rows, heads * D + pad, generator=g)).to(dt)
        self.q = wide[:, :heads * D].view(self.rows, heads, D)
        shape = (pages, kv_heads, page, D + pad) if heads_first else (pages, page, kv_heads, D + pad)
        self.k, self.v = ((s * torch.randn(shape, generator=g)).to(dt)[..., :D] for s in (size, 1.0))
        if heads_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.scale = D ** -0.5

    def on_device(self):
        def same_strides(x):
            y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
            return y.copy_(x)
        return [same_strides(x) for x in (self.q, self.k, self.v)] + [ints(self.start), ints(self.length), ints(self.table)]

    def check(self, **kw):
        q, k, v, st, ln, tb = self.on_device()
        out = torch.full(q.shape, 3.0, dtype=q.dtype, device="cuda")
        got = P.ttf_attend(q, k, v, st, ln, tb, self.scale, out=out, **kw)
        assert got is out and P.ttf_paged_status() == 0
        m = self.start[-1]
        assert (out[m:] == 3).all()
        ref, tol = attend_ref(self.q, self.k, self.v, self.start, self.length, self.table, self.scale, **kw)
        assert worst(out[:m].cpu(), ref[:m], tol[:m]) <= 1
        return out


# new, before, page, heads, kv_heads, D, dtype, mask
CASES = [
    ([1], [0], 16, 1, 1, 64, "bf16", {}),
    ([1], [0], 1, 4, 4, 128, "f32", {}),
    ([1], [700], 16, 32, 8, 128, "bf16", {}),
    ([1, 1, 1, 1, 1], [0, 1, 15, 16, 333], 16, 8, 2, 128, "bf16", {}),
    ([1, 1, 1], [200, 5, 64], 7, 6, 2, 64, "bf16", {}),
    ([1, 1], [500, 90], 48, 14, 2, 128, "bf16", dict(window=37)),
    ([1, 1], [300, 65], 32, 16, 1, 256, "bf16", {}),
    ([1, 1], [130, 65], 32, 20, 1, 96, "bf16", {}),
    ([2, 0, 7, 1], [40, 3, 100, 0], 32, 8, 8, 128, "bf16", {}),
    ([17, 5], [0, 61], 16, 8, 2, 80, "bf16", {}),
    ([64], [0], 64, 4, 1, 128, "bf16", {}),
    ([65, 31], [129, 0], 64, 8, 2, 128, "bf16", {}),
    ([200], [0], 64, 4, 2, 128, "bf16", {}),
    ([129], [300], 128, 4, 1, 64, "bf16", dict(causal=False)),
    ([130, 3, 77], [70, 400, 0], 256, 6, 2, 128, "bf16", dict(window=50)),
    ([90], [40], 128, 10, 2, 72, "bf16", dict(causal=False, window=33)),
    ([140], [300], 32, 7, 1, 120, "bf16", {}),
    ([33], [10], 16, 3, 3, 192, "bf16", {}),
    ([50, 1, 9], [13, 700, 0], 48, 4, 4, 72, "f32", dict(window=100)),
    ([33], [64], 16, 3, 1, 128, "f32", dict(causal=False)),
    ([5, 1], [40, 300], 5, 2, 1, 256, "f32", {}),
    ([6], [30], 16, 3, 1, 33, "f32", {}),
    ([6], [30], 16, 3, 1, 7, "bf16", {}),
    ([70], [30], 16, 3, 1, 66, "bf16", {}),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("heads_first", [False, True])
def test_attend(case, heads_first):
    *shape, mask = case
    Batch(*shape, heads_first=heads_first).check(**mask)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_strides_that_no_vector_fits(dtype, D):
    Batch([40, 1], [20, 90], 16, 4, 2, D, dtype, pad=1).check()
    Batch([40, 1], [20, 90], 16, 4, 2, D, dtype, pad=4).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[3, 9, 2], [1, 1, 1], [150, 200, 40]])
def test_rows_that_see_nothing(dtype, new):
    """a length below the number of new rows: the rows before the cache are zero; no slot at all; with and without a mask"""
    b = Batch(new, [0, 0, 0], 16, 4, 2, 64, dtype)
    b.length = [new[0] - 1, new[1] // 2, 0]
    for kw in (dict(), dict(causal=False), dict(window=1)):
        out = b.check(**kw)
        assert (out[0] == 0).all() and (out[b.start[2]:b.start[3]] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,before", [([1, 1], [37, 200]), ([70, 150], [37, 200])])
def test_slots_that_nobody_sees_may_hold_anything(dtype, new, before):
    b = Batch(new, before, 32, 4, 2, 128, dtype)
    q, k, v, st, ln, tb = b.on_device()
    clean = P.ttf_attend(q, k, v, st, ln, tb, b.scale, window=20, out=torch.zeros_like(q))
    k2, v2 = torch.full_like(k, float("nan")), torch.full_like(v, float("inf"))
    for s, n in enumerate(b.length):                        # only what some row sees is a number
        for slot in range(max(0, n - b.new[s] - 19), n):
            g, r = b.table[s][slot // 32], slot % 32
            k2[g, r], v2[g, r] = k[g, r], v[g, r]
    got = P.ttf_attend(q, k2, v2, st, ln, tb, b.scale, window=20, out=torch.zeros_like(q))
    assert torch.equal(got, clean)


@pytest.mark.parametrize("new", [1, 200])
def test_large_scores_do_not_overflow(new):
    b = Batch([new], [300], 16, 8, 2, 128, size=30.0)
    b.check()
    b.scale = -b.scale
    b.check()
    b.scale = 0.0
    b.check()


def test_one_row_of_lowest_scores():
    """keys that drive every score to the type's lowest finite values: weights are those of the differences"""
    b = Batch([1, 130], [40, 40], 16, 2, 1, 64)
    b.q[:] = 0
    b.q[..., 0] = 2.0 ** 60
    b.k[:] = 0
    b.k[..., 0] = -(2.0 ** 60)
    b.scale = 1.0
    out = b.check()
    assert torch.isfinite(out).all()


def test_new_rows_in_any_mixture_equal_one_by_one():
    b = Batch([1, 64, 3, 300, 1], [500, 0, 40, 77, 0], 64, 8, 2, 128)
    out = b.check()
    q, k, v, st, ln, tb = b.on_device()
    for s in range(5):
        one = P.ttf_attend(q[b.start[s]:b.start[s + 1]].contiguous(), k, v, ints([0, b.new[s]]), ln[s:s + 1], tb[s:s + 1], b.scale)
        a, c = out[b.start[s]:b.start[s + 1]].float(), one.float()
        assert float((a - c).abs().max()) <= 4 * 2.0 ** -8 * float(a.abs().max())


def test_deterministic_and_another_stream():
    b = Batch([1, 64, 3], [500, 0, 40], 16, 8, 2, 128)
    args = b.on_device()
    a = P.ttf_attend(*args, b.scale, out=torch.zeros_like(args[0]))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    c = P.ttf_attend(*args, b.scale, out=torch.zeros_like(args[0]), stream=st)
    st.synchronize()
    assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 70, 200])
def test_bad_metadata_is_reported_and_reads_nothing_outside(dtype, new):
    b = Batch([new, new], [100, 40], 32, 8, 2, 64, dtype)
    q, k, v, st, ln, tb = b.on_device()
    good = P.ttf_attend(q, k, v, st, ln, tb, b.scale)
    assert P.ttf_paged_status() == 0

    def bad(start=None, length=None, table=None):
        out = P.ttf_attend(q, k, v, st if start is None else ints(start), ln if length is None else ints(length),
                           tb if table is None else ints(table), b.scale)
        assert P.ttf_paged_status() == P.TTF_ERR_BOUNDS
        assert torch.equal(out[:new], good[:new])           # the other sequence is not affected

    for page in (k.shape[0], -1, 2**31 - 1, -2**31):
        t = [list(r) for r in b.table]
        t[1][0] = page
        bad(table=t)
    bad(length=[b.length[0], 32 * len(b.table[0]) + 1])
    bad(length=[b.length[0], -1])
    bad(start=[0, new, b.rows + 1])
    bad(start=[0, new, new - 1])
    assert torch.equal(P.ttf_attend(q, k, v, st, ln, tb, b.scale)[:2 * new], good[:2 * new]) and P.ttf_paged_status() == 0


def test_offsets_beyond_32_bits():
    page, hk, D = 256, 8, 128
    pages = (1 << 32) // (page * hk * D) + 2
    big = torch.empty((pages, page, hk, D), dtype=torch.bfloat16, device="cuda")
    for new in (1, 150):
        b = Batch([new], [200], page, 8, hk, D)
        last = len(b.table[0])
        q, k, v, st, ln, _ = b.on_device()
        at = [pages - 1 - i for i in range(last)]
        for i, g in enumerate(at):
            big[g].copy_(k[b.table[0][i]])
        got = P.ttf_attend(q, big, big, st, ln, ints([at]), b.scale)
        ref = P.ttf_attend(q, k, k, st, ln, ints(b.table), b.scale)
        assert torch.equal(got[:new], ref[:new])
