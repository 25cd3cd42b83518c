"""Which rows of a call are new tokens, and what is reported of sequences that do not fit: ttf_cache_append says the same of the
arrays as ttf_attend and include/ttf.h."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import ints, rotate_ref, worst

pytestmark = pytest.mark.gpu

HK, D, PAGE = 1, 32, 4
OK, BOUNDS = 0, P.TTF_ERR_BOUNDS

# start, length (page b of the cache is page 0 of sequence b), rows that are stored, status
CASES = {
    "as it should be": ([0, 4, 8], [4, 4], range(8), OK),
    "the last start lies below the one before": ([0, 4, 3], [4, 4], range(4), BOUNDS),
    "a negative last start": ([0, 4, -2], [4, 4], range(4), BOUNDS),
    "a negative first start": ([-1, 4, 8], [4, 4], range(4, 8), BOUNDS),
    "rows beyond the arrays, then a sequence that goes back": ([0, 9, 8], [4, 4], [], BOUNDS),
    "no new rows and a negative length": ([0, 4, 4], [4, -1], range(4), BOUNDS),
    "no new rows and a length beyond the table": ([0, 0, 4], [99, 4], range(4), BOUNDS),
    "rows before the first sequence": ([2, 5, 8], [3, 3], range(2, 8), OK),
    "rows before the only sequence": ([7, 8], [4], [7], OK),
    "no rows at all": ([5, 5, 5], [4, 0], [], OK),
    "a sequence in the middle that goes back": ([0, 4, 3, 8], [4, 4, 4], [0, 1, 2, 4, 5, 6, 7], BOUNDS),
}


def inputs(rows, seed=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(rows, h, D, generator=g) for h in (HK, HK, 2)]


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("turned", [False, True])
def test_rows_and_reports(name, turned):
    start, length, stored, status = CASES[name]
    k, v, q = inputs(8)
    seqs = len(length)
    kc, vc = (torch.full((seqs, PAGE, HK, D), 5.0, device="cuda") for _ in range(2))
    table = ints([[b] for b in range(seqs)])
    oq = torch.full((8, 2, D), 5.0, device="cuda")
    pos, freq = torch.arange(8, dtype=torch.int32), torch.rand(D // 2, generator=torch.Generator().manual_seed(2))
    more = dict(positions=pos.cuda(), freq=freq.cuda(), q=q.cuda(), out_q=oq) if turned else {}
    P.ttf_cache_append(k.cuda(), v.cuda(), kc, vc, ints(start), ints(length), table, **more)
    assert P.ttf_paged_status() == status
    P.ttf_attend(q.cuda(), kc, vc, ints(start), ints(length), table, 1.0, out=torch.zeros(8, 2, D, device="cuda"))
    assert P.ttf_paged_status() == status                   # (the two agree)
    ref, tol = rotate_ref(k, pos, freq) if turned else (k.double(), torch.zeros(8, HK, D, dtype=torch.float64))
    refq, tolq = rotate_ref(q, pos, freq)
    for row in stored:
        b = max(s for s in range(seqs) if start[s] <= row < start[s + 1])
        slot = length[b] - start[b + 1] + row
        if len([s for s in range(seqs) if start[s] <= row < start[s + 1]]) == 1:
            assert torch.equal(vc[b, slot].cpu(), v[row])
            assert worst(kc[b, slot].cpu(), ref[row], tol[row]) <= 1
        if turned:
            assert worst(oq[row].cpu(), refq[row], tolq[row]) <= 1
    claimed = sum(1 for r in range(8) if any(start[s] <= r < start[s + 1] for s in range(seqs)))
    assert int((vc != 5.0).all(-1).sum()) <= max(claimed, len(stored))
    if turned:                                              # rows that belong to no sequence are left as they were
        for row in range(8):
            if not any(start[s] <= row < start[s + 1] for s in range(seqs)):
                assert (oq[row] == 5.0).all()


@pytest.mark.parametrize("seqs", [31, 32, 33, 70, 200])
def test_one_bad_sequence_among_many(seqs):
    """rows of all others are stored, whatever lane looks a sequence up; three rows before the first one stay out"""
    first = 3
    rows = first + seqs
    k, v, _ = inputs(rows)
    start = [first + i for i in range(seqs + 1)]
    for bad in (0, seqs // 2, seqs - 1):
        length = [1 + i % PAGE for i in range(seqs)]
        length[bad] = PAGE + 1
        kc, vc = (torch.full((seqs, PAGE, HK, D), 5.0, device="cuda") for _ in range(2))
        P.ttf_cache_append(k.cuda(), v.cuda(), kc, vc, ints(start), ints(length), ints([[b] for b in range(seqs)]))
        assert P.ttf_paged_status() == BOUNDS
        want_k, want_v = (torch.full((seqs, PAGE, HK, D), 5.0) for _ in range(2))
        for b in range(seqs):
            if b != bad:
                want_k[b, length[b] - 1], want_v[b, length[b] - 1] = k[first + b], v[first + b]
        assert torch.equal(kc.cpu(), want_k) and torch.equal(vc.cpu(), want_v)
