"""ttf_attend of fp32 heads: the form for few rows (a CTA per 8) and the one for many (a CTA per 64), with the slots shared by a
cluster and not, against the definition in 64 bits."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import attend_ref, worst
from tests.test_gpu_attend import Batch

pytestmark = pytest.mark.gpu

# new, before, page, heads, kv_heads, D, mask
CASES = [
    ([1], [5000], 16, 8, 1, 128, {}),                      # few rows, a cluster of 16
    ([1] * 40, [7 * i for i in range(40)], 24, 16, 8, 64, {}),
    ([1, 1, 2], [900, 31, 0], 1, 10, 2, 256, {}),
    ([9, 1], [70, 2], 33, 4, 4, 132, dict(window=16)),
    ([3, 0, 8], [100, 9, 0], 16, 7, 1, 4, dict(causal=False)),
    ([100], [1900], 64, 4, 2, 128, {}),                    # many rows, a cluster of 8
    ([65, 129], [0, 300], 7, 6, 2, 192, {}),
    ([90, 40], [100, 5], 48, 2, 1, 256, dict(window=40)),
    ([700], [0], 32, 3, 3, 72, dict(causal=False)),
    ([33, 200, 0, 1], [64, 31, 5, 0], 16, 8, 2, 36, {}),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("heads_first", [False, True])
def test_attend(case, heads_first):
    *shape, mask = case
    Batch(*shape, "f32", heads_first=heads_first, spare=0).check(**mask)


@pytest.mark.parametrize("new,D", [(5, 128), (5, 256), (80, 64), (80, 256)])
def test_what_a_row_does_not_see_may_be_seen_by_others(new, D):
    """the last two tokens' slots hold no numbers: only the last two rows may tell"""
    b = Batch([new], [50], 16, 4, 2, D, "f32", spare=0)
    q, k, v, st, ln, tb = b.on_device()
    clean = P.ttf_attend(q, k, v, st, ln, tb, b.scale, out=torch.zeros_like(q))
    for slot, x in ((50 + new - 1, float("nan")), (50 + new - 2, float("inf"))):
        g, r = b.table[0][slot // 16], slot % 16
        k[g, r], v[g, r] = x, x
    got = P.ttf_attend(q, k, v, st, ln, tb, b.scale, out=torch.zeros_like(q))
    assert torch.equal(got[:-2], clean[:-2]) and got[-2:].isnan().all()


@pytest.mark.parametrize("new", [1, 100])
def test_sums_over_many_slots_keep_their_digits(new):
    """Equal weights and values of one sign.  Every partial sum is at most n v; with chains of c terms, and m of them added,
    each addition is off by half a step of at most the whole sum, so the result is off by (c + m) half steps at the worst, and by
    about the root of that when their signs are mixed.  One chain over all 12001 slots drifts by more than 2^-24 * 64."""
    b = Batch([new], [12000], 64, 8 if new == 1 else 1, 1, 64, "f32", spare=0)
    b.k.zero_()
    b.v.abs_()
    q, k, v, st, ln, tb = b.on_device()
    got = P.ttf_attend(q, k, v, st, ln, tb, b.scale, out=torch.zeros_like(q))
    ref, _ = attend_ref(b.q, b.k, b.v, b.start, b.length, b.table, b.scale)
    ref = ref.double()
    assert ((got.cpu().double() - ref).abs() / ref).max() <= 32 * 2.0 ** -24


def test_strides_of_one_head_and_unaligned_rows():
    Batch([40, 1], [20, 90], 16, 4, 2, 64, "f32", pad=3).check()        # (no 16-byte pieces: the scalar form)
    Batch([4, 1], [20, 90], 16, 4, 2, 64, "f32", pad=8).check()
    Batch([140], [90], 16, 4, 2, 64, "f32", pad=8).check()
