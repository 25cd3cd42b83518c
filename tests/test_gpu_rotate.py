"""ttf_rotate and ttf_cache_append against the definitions in 64 bits (tests/paged.py)."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import DTYPES, ints, rotate_ref, spread_pages, starts, worst

pytestmark = pytest.mark.gpu


def table_of(rot, theta=1e4):
    j = torch.arange(rot // 2, dtype=torch.float64)
    return (theta ** (-2 * j / max(rot, 1))).float()


def sections_of(rot, axes):
    pairs = rot // 2
    if axes == 1:
        return None
    h = pairs // (axes + 1)
    return (pairs - (axes - 1) * h,) + (h,) * (axes - 1)


# rows, query heads, key heads, D, rot, interleaved, axes, cyclic, norm, dtype, far
CASES = [
    (1, 1, 1, 128, 128, False, 3, True, True, "bf16", 0),
    (5, 32, 8, 128, 128, False, 3, True, True, "bf16", 35),
    (300, 16, 2, 128, 128, False, 3, False, True, "bf16", 35),
    (7, 4, 2, 64, 64, True, 1, False, True, "bf16", 1000),
    (9, 6, 3, 96, 48, False, 2, True, False, "bf16", 7),
    (9, 3, 3, 80, 40, True, 2, False, True, "f32", 7),
    (1153, 3, 1, 72, 36, True, 1, False, False, "f32", 1_000_000),
    (6, 2, 1, 72, 36, False, 1, False, True, "bf16", 50_000),       # halves of 18 pairs: two channels at a time
    (6, 2, 1, 256, 254, False, 3, True, True, "bf16", 5),           # halves of 127 pairs: one at a time, four items per lane
    (6, 2, 1, 256, 252, False, 1, False, True, "f32", 5),
    (4, 3, 2, 7, 4, False, 1, False, True, "f32", 3),               # odd heads
    (4, 3, 2, 33, 10, True, 1, False, True, "bf16", 3),
    (4, 3, 2, 1, 0, False, 1, False, True, "f32", 3),               # a norm alone
    (2000, 1, 1, 16, 16, False, 1, False, True, "bf16", 2_000_000_000),
    (3, 70, 70, 128, 128, False, 1, False, True, "f32", 1 << 30),
]


def inputs(case, seed=0, pad=0):
    rows, hq, hk, D, rot, inter, axes, cyc, norm, dt, far = case
    g = torch.Generator().manual_seed(seed + rows + D)
    dtype = DTYPES[dt]
    rand = lambda *s: torch.randn(s, generator=g).to(dtype)
    wide = rand(rows, (hq + hk) * D + pad)                  # heads as parts of a wider row
    q, k = wide[:, :hq * D].view(rows, hq, D), wide[:, hq * D:(hq + hk) * D].view(rows, hk, D)
    pos = (torch.randint(0, 300, (rows, axes), generator=g) + far).int()
    turn = dict(rot_dim=rot, interleaved=inter, sections=sections_of(rot, axes), cyclic=cyc, factor=1.25 if inter else 1.0)
    qw = (1 + rand(D) / 4) if norm else None
    kw = (1 + rand(D) / 4) if norm else None
    return wide, q, k, pos, table_of(rot), qw, kw, turn


def cuda(x):
    return None if x is None else x.cuda()


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("pad", [0, 1])
def test_rotate(case, pad):
    rows, hq, hk, D = case[:4]
    wide, q, k, pos, freq, qw, kw, turn = inputs(case, pad=pad)
    dev = wide.cuda()
    dq, dk = dev[:, :hq * D].view(rows, hq, D), dev[:, hq * D:(hq + hk) * D].view(rows, hk, D)
    oq, ok = P.ttf_rotate(dq, dk, pos.cuda(), freq.cuda(), q_weight=cuda(qw), k_weight=cuda(kw), **turn)
    for got, x, w in ((oq, q, qw), (ok, k, kw)):
        ref, tol = rotate_ref(x, pos, freq, w, **turn)
        assert worst(got.cpu(), ref, tol) <= 1
    # in place: the same bits
    P.ttf_rotate(dq, dk, pos.cuda(), freq.cuda(), q_weight=cuda(qw), k_weight=cuda(kw), out_q=dq, out_k=dk, **turn)
    assert torch.equal(dq, oq) and torch.equal(dk, ok)
    assert P.ttf_paged_status() == 0


def test_rotate_one_of_the_two_and_a_count_on_the_device():
    case = CASES[2]
    rows, hq, hk, D = case[:4]
    _, q, k, pos, freq, qw, kw, turn = inputs(case)
    full, _ = P.ttf_rotate(q.cuda(), None, pos.cuda(), freq.cuda(), q_weight=qw.cuda(), **turn)
    both, fk = P.ttf_rotate(q.cuda(), k.cuda(), pos.cuda(), freq.cuda(), q_weight=qw.cuda(), **turn)
    assert torch.equal(full, both)                          # (keys without a weight beside queries with one)
    ref, tol = rotate_ref(k, pos, freq, None, **turn)
    assert worst(fk.cpu(), ref, tol) <= 1
    for n in (0, 1, 149, rows, rows + 7, -3):
        oq, ok = torch.full_like(full, 7), torch.full_like(fk, 7)
        P.ttf_rotate(q.cuda(), k.cuda(), pos.cuda(), freq.cuda(), q_weight=qw.cuda(), count=ints([n]), out_q=oq, out_k=ok, **turn)
        m = min(max(n, 0), rows)
        assert torch.equal(oq[:m], full[:m]) and torch.equal(ok[:m], fk[:m])
        assert (oq[m:] == 7).all() and (ok[m:] == 7).all()


def test_far_positions_keep_their_turns():
    """neighbouring positions near 2^31 differ by exactly one step of the fastest pair"""
    pos = torch.tensor([2**31 - 2, 2**31 - 1], dtype=torch.int32)
    x = torch.tensor([[[1.0, 0.0]], [[1.0, 0.0]]])
    freq = torch.tensor([1.0])
    got = P.ttf_rotate(x.cuda(), None, pos.cuda(), freq.cuda())[0].cpu()
    ref, tol = rotate_ref(x, pos, freq)
    assert worst(got, ref, tol) <= 1


def test_nan_and_infinity_stay_in_their_head():
    case = CASES[1]
    _, q, k, pos, freq, qw, kw, turn = inputs(case)
    clean = P.ttf_rotate(q.cuda(), k.cuda(), pos.cuda(), freq.cuda(), q_weight=qw.cuda(), k_weight=kw.cuda(), **turn)
    q, k = q.clone(), k.clone()
    q[2, 3, 5] = float("nan")
    k[4, 1, 0] = float("inf")
    oq, ok = P.ttf_rotate(q.cuda(), k.cuda(), pos.cuda(), freq.cuda(), q_weight=qw.cuda(), k_weight=kw.cuda(), **turn)
    assert oq[2, 3].isnan().all()
    oq[2, 3], ok[4, 1] = clean[0][2, 3], clean[1][4, 1]
    assert torch.equal(oq, clean[0]) and torch.equal(ok, clean[1])


# new tokens and lengths before them, page size, [pages, heads, page, D] in memory?
BATCHES = [
    ([1], [0], 1, False),
    ([1, 1, 1], [0, 31, 32], 16, False),
    ([5, 0, 70, 1], [0, 9, 100, 63], 48, True),
    ([200], [35], 64, True),
    ([1] * 70, list(range(70)), 7, False),
]


@pytest.mark.parametrize("case", [CASES[1], CASES[4], CASES[5], CASES[7], CASES[11]], ids=str)
@pytest.mark.parametrize("batch", BATCHES, ids=str)
@pytest.mark.parametrize("with_q", [True, False])
def test_append(case, batch, with_q):
    new, before, page, heads_first = batch
    hq, hk, D = case[1:4]
    spare = 3
    rows = sum(new) + spare
    case = (rows,) + case[1:]
    _, q, k, pos, freq, qw, kw, turn = inputs(case)
    g = torch.Generator().manual_seed(5)
    v = torch.randn(rows, hk, D, generator=g).to(k.dtype)
    length = [a + b for a, b in zip(new, before)]
    table, pages = spread_pages(length, page, g)
    shape = (pages, hk, page, D) if heads_first else (pages, page, hk, D)
    kc, vc = (torch.full(shape, 9, dtype=k.dtype, device="cuda") for _ in range(2))
    kv, vv = (c.transpose(1, 2) if heads_first else c for c in (kc, vc))
    oq = torch.full((rows, hq, D), 9, dtype=k.dtype, device="cuda")
    args = dict(q=q.cuda(), out_q=oq) if with_q else {}
    got = P.ttf_cache_append(k.cuda(), v.cuda(), kv, vv, ints(starts(new)), ints(length), ints(table), pos.cuda(), freq.cuda(),
                             q_weight=cuda(qw), k_weight=cuda(kw), **args, **turn)
    assert (got is oq) if with_q else got is None
    assert P.ttf_paged_status() == 0
    ref, tol = rotate_ref(k, pos, freq, kw, **turn)
    where = {}
    st = starts(new)
    for b, n in enumerate(new):
        for i in range(n):
            s = length[b] - n + i
            where[st[b] + i] = (table[b][s // page], s % page)
    kv, vv = kv.cpu(), vv.cpu()
    for row, (g_, r_) in where.items():
        assert torch.equal(vv[g_, r_], v[row])
        assert worst(kv[g_, r_], ref[row], tol[row]) <= 1
        kv[g_, r_] = vv[g_, r_] = 9
    assert (kv == 9).all() and (vv == 9).all()              # nothing else was written
    if with_q:
        ref, tol = rotate_ref(q, pos, freq, qw, **turn)
        m = sum(new)
        assert worst(oq[:m].cpu(), ref[:m], tol[:m]) <= 1
        assert (oq[m:] == 9).all()


def test_append_without_rotation_copies():
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(6, 2, 40, generator=g).bfloat16().cuda() for _ in range(2))
    kc, vc = (torch.zeros(4, 4, 2, 40, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    P.ttf_cache_append(k, v, kc, vc, ints([0, 6]), ints([9]), ints([[2, 0, 3]]))
    assert torch.equal(kc[2, 3], k[0]) and torch.equal(kc[0], k[1:5]) and torch.equal(kc[3, 0], k[5])
    assert torch.equal(vc[2, 3], v[0]) and torch.equal(vc[0], v[1:5]) and torch.equal(vc[3, 0], v[5])
    assert (kc[1] == 0).all() and (kc[3, 1:] == 0).all() and (kc[2, :3] == 0).all()


def test_keys_and_values_interleaved_in_one_array():
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(5, 3, 64, generator=g).bfloat16().cuda() for _ in range(2))
    both = torch.zeros(4, 2, 8, 3, 64, dtype=torch.bfloat16, device="cuda")
    P.ttf_cache_append(k, v, both[:, 0], both[:, 1], ints([0, 5]), ints([5]), ints([[3]]))
    assert torch.equal(both[3, 0, :5], k) and torch.equal(both[3, 1, :5], v) and (both[:3] == 0).all()


def test_bad_metadata_is_reported_and_nothing_outside_is_touched():
    """Pages that are not there, lengths beyond the table, rows beyond the arrays: the sequence's tokens are left out, the
    others are stored, and the status says so once."""
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(8, 1, 32, generator=g).cuda() for _ in range(2))

    def call(start, length, table):
        kc, vc = (torch.full((3, 4, 1, 32), 5.0, device="cuda") for _ in range(2))
        P.ttf_cache_append(k, v, kc, vc, ints(start), ints(length), ints(table))
        assert torch.equal(kc == 5.0, vc == 5.0)
        return P.ttf_paged_status(), (kc != 5.0).all(-1).all(-1).sum().item()

    assert call([0, 4, 8], [4, 4], [[0], [1]]) == (0, 8)
    assert P.ttf_paged_status() == 0
    for bad in (3, -1, 2**31 - 1, -2**31):
        assert call([0, 4, 8], [4, 4], [[0], [bad]]) == (P.TTF_ERR_BOUNDS, 4)
    assert call([0, 4, 8], [4, 5], [[0], [1]]) == (P.TTF_ERR_BOUNDS, 4)          # beyond the table
    assert call([0, 4, 8], [4, -1], [[0], [1]]) == (P.TTF_ERR_BOUNDS, 4)
    assert call([0, 4, 9], [4, 4], [[0], [1]]) == (P.TTF_ERR_BOUNDS, 4)          # rows beyond the arrays
    assert call([0, 4, 8], [4, 2], [[0], [1]]) == (0, 6)                         # two tokens before the cache: no slot
    assert call([0, 4, 8], [4, 4], [[0], [1]]) == (0, 8)


def test_offsets_beyond_32_bits():
    """a cache of more than 2^32 elements: its last page"""
    page, hk, D = 256, 8, 128
    pages = (1 << 32) // (page * hk * D) + 2
    kc = torch.empty((pages, page, hk, D), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(4)
    k = torch.randn(3, hk, D, generator=g).bfloat16().cuda()
    v = torch.randn(3, hk, D, generator=g).bfloat16().cuda()
    kc[pages - 1].zero_()
    kc[0].zero_()
    P.ttf_cache_append(k, v, kc[1:], kc[:-1], ints([0, 3]), ints([3]), ints([[pages - 2]]))
    assert torch.equal(kc[pages - 1, :3], k) and (kc[pages - 1, 3:] == 0).all()
    assert torch.equal(kc[pages - 2, :3], v)
    assert (kc[0] == 0).all()
