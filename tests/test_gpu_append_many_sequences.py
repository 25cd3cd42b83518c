"""ttf_cache_append over more sequences than a warp has lanes: empty ones among them, starts that go back somewhere, rows that only
sequences before such a start claim."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import ints

pytestmark = pytest.mark.gpu

HK, D, PAGE = 2, 16, 4


def run(start, length, rows, seed=1):
    """every sequence has one page of its own; what is stored against a plain loop over the sequences (bad ones are left out)"""
    g = torch.Generator().manual_seed(seed)
    seqs = len(length)
    k, v = (torch.randn(rows, HK, D, generator=g) for _ in range(2))
    kc, vc = (torch.full((seqs, PAGE, HK, D), 5.0, device="cuda") for _ in range(2))
    P.ttf_cache_append(k.cuda(), v.cuda(), kc, vc, ints(start), ints(length), ints(list(range(seqs))).view(-1, 1))
    want_k, want_v = (torch.full((seqs, PAGE, HK, D), 5.0) for _ in range(2))
    bad, claimed = False, {}
    for b in range(seqs):
        ok = 0 <= start[b] <= start[b + 1] <= rows and 0 <= length[b] <= PAGE
        bad = bad or not ok
        for i in range(max(0, start[b]), min(start[b + 1], rows)) if start[b] >= 0 and start[b + 1] <= rows else []:
            claimed.setdefault(i, []).append(b)
            slot = length[b] - start[b + 1] + i
            if ok and slot >= 0:
                want_k[b, slot], want_v[b, slot] = k[i], v[i]
    got_k, got_v = kc.cpu(), vc.cpu()
    for i, by in claimed.items():                           # rows of two sequences: undefined
        if len(by) > 1:
            for b in by:
                slot = length[b] - start[b + 1] + i
                if 0 <= slot < PAGE:
                    got_k[b, slot], got_v[b, slot] = want_k[b, slot], want_v[b, slot]
    assert torch.equal(got_k, want_k) and torch.equal(got_v, want_v)
    assert P.ttf_paged_status() == (P.TTF_ERR_BOUNDS if bad else 0)


def spread(seqs, seed, first=0):
    g = torch.Generator().manual_seed(seed)
    new = torch.randint(0, PAGE + 1, (seqs,), generator=g).tolist()
    start = [first]
    for n in new:
        start.append(start[-1] + n)
    return start, [n + int(torch.randint(0, PAGE + 1 - n, (1,), generator=g)) for n in new]


@pytest.mark.parametrize("seqs", [31, 32, 33, 63, 64, 65, 100, 1000, 1024, 1025, 3000])
@pytest.mark.parametrize("first", [0, 7])
def test_all_as_it_should_be(seqs, first):
    start, length = spread(seqs, seqs, first)
    run(start, length, start[-1] + 3)


@pytest.mark.parametrize("seqs", [33, 100, 1000, 1500])
def test_many_empty_ones(seqs):
    start = [0] * (seqs // 2) + [2] * (seqs - seqs // 2) + [4]
    run(start, [PAGE] * seqs, 6)


@pytest.mark.parametrize("seqs", [20, 33, 64, 100, 1000, 1100])
@pytest.mark.parametrize("where", [0.0, 0.3, 0.5, 0.97])
def test_a_start_that_goes_back(seqs, where):
    start, length = spread(seqs, seqs + 1)
    at = 1 + int(where * (seqs - 2))
    start[at] = max(0, start[at] // 3 - 1)                  # claims rows of others, and its own sequence goes back
    run(start, length, start[-1])


@pytest.mark.parametrize("seqs", [5, 33, 100, 1000])
@pytest.mark.parametrize("last", [-5, 0, 3, 10**9])
def test_a_last_start_that_is_out_of_place(seqs, last):
    """the rows that the other sequences claim lie beyond it"""
    start, length = spread(seqs, seqs + 2)
    rows = start[-1] + 2
    start[-1] = last
    run(start, length, rows)
