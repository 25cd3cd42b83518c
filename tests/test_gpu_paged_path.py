"""The way of a clip's tokens from ttf_compress to attention and on to decoding: ttf_rotate, ttf_cache_append and ttf_attend with
counts, positions and lengths that only the device knows; the same captured and replayed, on several streams at once, and the
bounded waits of the kernels."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import binding as B
from tests.paged import attend_ref, ints, rotate_ref, worst
from tests.parity import to_device
from tests.test_gpu_attend import Batch
from tests.test_gpu_parity import corr_clip

pytestmark = pytest.mark.gpu

F, H, W, C = 6, 6, 7, 256
HQ, HK, D, PAGE = 8, 2, 64, 16
SECTIONS = (12, 10, 10)
TEXT = 5                                                    # tokens of a prompt before the clip


class Layer:
    """random projections and norms of one layer, and a cache"""

    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.proj = (torch.randn(C, (HQ + 2 * HK) * D, generator=g) / C ** 0.5).bfloat16().cuda()
        self.qw, self.kw = ((1 + torch.randn(D, generator=g) / 5).bfloat16().cuda() for _ in range(2))
        self.freq = (1e4 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).float().cuda()
        self.pages = 40
        self.table = torch.randperm(self.pages, generator=g)[:24].int().view(1, 24).cuda()
        self.k = torch.zeros(self.pages, PAGE, HK, D, dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros_like(self.k)

    def turn(self):
        return dict(q_weight=self.qw, k_weight=self.kw, sections=SECTIONS, cyclic=True)

    def attend(self, x, pos, start, length, q_out, out):
        """x [rows, C]: projection, append with rotation, attention"""
        qkv = (x @ self.proj).view(x.shape[0], HQ + 2 * HK, D)
        P.ttf_cache_append(qkv[:, HQ:HQ + HK], qkv[:, HQ + HK:], self.k, self.v, start, length, self.table, pos, self.freq,
                           q=qkv[:, :HQ], out_q=q_out, **self.turn())
        P.ttf_attend(q_out, self.k, self.v, start, length, self.table, D ** -0.5, out=out)
        return qkv


def step(layer, clip, bufs):
    """compress a clip, then prompt text and clip as one chunk of TEXT + L' new tokens; then one decoded token"""
    tok, cnt, pos, x, pos_all, start, length, q_out, out, q1, o1 = bufs
    P.ttf_compress(clip, 1, 0.7, tok, cnt, pos, pos_base=TEXT)
    x[TEXT:].copy_(tok)
    pos_all[TEXT:].copy_(pos)
    start[1:].copy_(cnt + TEXT)
    length.copy_(cnt + TEXT)
    qkv = layer.attend(x, pos_all, start, length, q_out, out)
    # the next token: behind the clip in the cache, at position L' + T
    one = torch.arange(2, dtype=torch.int32, device="cuda")
    dec_pos = (cnt + TEXT).view(1, 1).repeat(1, 3).contiguous()
    layer.attend(x[:1], dec_pos, one, length + 1, q1, o1)
    return qkv


def buffers(seed):
    g = torch.Generator().manual_seed(seed)
    n = F * H * W
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    x = bf(n + TEXT, C)
    x[:TEXT] = torch.randn(TEXT, C, generator=g).bfloat16().cuda()
    pos_all = torch.zeros(n + TEXT, 3, dtype=torch.int32, device="cuda")
    pos_all[:TEXT] = torch.arange(TEXT, dtype=torch.int32, device="cuda").view(TEXT, 1)
    return (bf(n, C), ints([0]), torch.zeros(n, 3, dtype=torch.int32, device="cuda"), x, pos_all, ints([0, 0]), ints([0]),
            bf(n + TEXT, HQ, D), bf(n + TEXT, HQ, D), bf(1, HQ, D), bf(1, HQ, D))


def check(layer, bufs, qkv):
    tok, cnt, pos, x, pos_all, start, length, q_out, out, q1, o1 = bufs
    n = int(cnt) + TEXT
    assert H * W + TEXT < n < F * H * W + TEXT              # something was fused, something kept
    qkv = qkv.cpu()
    args = dict(sections=SECTIONS, cyclic=True)
    ref, tol = rotate_ref(qkv[:n, :HQ], pos_all[:n].cpu(), layer.freq.cpu(), layer.qw.cpu(), **args)
    assert worst(q_out[:n].cpu(), ref, tol) <= 1
    refk, tolk = rotate_ref(qkv[:n, HQ:HQ + HK], pos_all[:n].cpu(), layer.freq.cpu(), layer.kw.cpu(), **args)
    table = layer.table.cpu()[0].tolist()
    k, v = layer.k.cpu(), layer.v.cpu()
    for i in range(n):
        g, r = table[i // PAGE], i % PAGE
        assert worst(k[g, r], refk[i], tolk[i]) <= 1
        assert torch.equal(v[g, r], qkv[i, HQ + HK:])
    ref, tol = attend_ref(q_out[:n].cpu(), k, v, [0, n], [n], [table], D ** -0.5)
    assert worst(out[:n].cpu(), ref, tol) <= 1
    assert (out[n:] == 0).all() and (q_out[n:] == 0).all()
    ref, tol = attend_ref(q1.cpu(), k, v, [0, 1], [n + 1], [table], D ** -0.5)
    assert worst(o1.cpu(), ref, tol) <= 1


def clip_of(seed):
    return to_device(corr_clip(F, H, W, C, seed=seed, dtype="bf16"))


def test_clip_to_decoded_token():
    layer, bufs = Layer(1), buffers(1)
    qkv = step(layer, clip_of(3), bufs)
    torch.cuda.synchronize()
    check(layer, bufs, qkv)
    assert P.ttf_paged_status() == B.TTF_OK


def test_the_same_captured_and_replayed_with_other_clips():
    """one graph, replayed with clips of other counts: lengths and rows follow the device"""
    layer, bufs, clip = Layer(2), buffers(2), clip_of(3)
    step(layer, clip, bufs)                                 # (scratch of ttf_compress, outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(layer, clip, bufs)                             # the side stream's own scratch
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        qkv = step(layer, clip, bufs)
    counts = set()
    for seed in (11, 12, 13):
        clip.copy_(clip_of(seed))
        for b in (bufs[7], bufs[8]):
            b.zero_()
        layer.k.zero_(); layer.v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(layer, bufs, qkv)
        counts.add(int(bufs[1]))
    assert len(counts) > 1 and P.ttf_paged_status() == B.TTF_OK


def test_several_streams_at_once():
    """calls on different streams share nothing: every one gives the bits it gives alone"""
    shapes = [([1] * 9, [70 * i for i in range(9)]), ([200, 3], [50, 400]), ([1], [3000]), ([65], [700])]
    batches = [Batch(new, before, 16, 8, 2, 128, seed=i) for i, (new, before) in enumerate(shapes)]
    args = [b.on_device() for b in batches]
    alone = [P.ttf_attend(*a, b.scale, out=torch.zeros_like(a[0])) for a, b in zip(args, batches)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    outs = [torch.zeros_like(a[0]) for a in args]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, a, b, o in zip(streams, args, batches, outs):
            P.ttf_attend(*a, b.scale, out=o, stream=st)
    torch.cuda.synchronize()
    for x, y in zip(alone, outs):
        assert torch.equal(x, y)


def test_two_graphs_replayed_at_once():
    """graphs captured on one stream and replayed on two"""
    b = [Batch([150], [900], 32, 8, 2, 128, seed=s) for s in (1, 2)]
    args = [x.on_device() for x in b]
    ref = [P.ttf_attend(*a, x.scale, out=torch.zeros_like(a[0])) for a, x in zip(args, b)]
    outs = [torch.zeros_like(a[0]) for a in args]
    graphs = []
    for a, x, o in zip(args, b, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            P.ttf_attend(*a, x.scale, out=o)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in b]
    torch.cuda.synchronize()
    for _ in range(10):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for x, y in zip(ref, outs):
        assert torch.equal(x, y)


def test_sequences_may_share_pages():
    """a prompt that several requests have in common lies in the cache once"""
    b = Batch([1, 1, 40], [96, 96, 96], 32, 4, 1, 64)
    for s in (1, 2):
        b.table[s][:3] = b.table[0][:3]
    b.check()


def test_a_row_of_the_table_may_be_part_of_a_wider_one():
    b = Batch([1, 70], [200, 35], 16, 4, 2, 128)
    q, k, v, st, ln, tb = b.on_device()
    ref = P.ttf_attend(q, k, v, st, ln, tb, b.scale, out=torch.zeros_like(q))
    wide = torch.full((2, tb.shape[1] + 5), 2**30, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + tb.shape[1]] = tb
    got = P.ttf_attend(q, k, v, st, ln, wide[:, 2:2 + tb.shape[1]], b.scale, out=torch.zeros_like(q))
    assert torch.equal(got, ref)


@pytest.mark.parametrize("new,before", [([1, 1], [300, 40]), ([150, 90], [200, 0]), ([130], [4000])])
def test_waits_run_out_and_the_next_call_is_clean(new, before):
    """the hook makes every copy barrier expect more than its copies deliver: the kernels report, free their tensor memory and
    return; then everything is as before"""
    b = Batch(new, before, 16, 8, 2, 128)
    args = b.on_device()
    ref = P.ttf_attend(*args, b.scale, out=torch.zeros_like(args[0]))
    assert P.ttf_paged_status() == B.TTF_OK
    P.ttf_debug_set_wait(32, 16)
    try:
        P.ttf_attend(*args, b.scale, out=torch.zeros_like(args[0]))
        assert P.ttf_paged_status() == B.TTF_ERR_TIMEOUT
    finally:
        P.ttf_debug_set_wait()
    got = P.ttf_attend(*args, b.scale, out=torch.zeros_like(args[0]))
    assert P.ttf_paged_status() == B.TTF_OK and torch.equal(got, ref)


@pytest.mark.parametrize("seed", range(24))
def test_drawn_sizes(seed):
    """batches, pages, heads and masks as they come"""
    import random
    rng = random.Random(seed)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    seqs = log(1, 40)
    dtype = "f32" if seed % 6 == 5 else "bf16"
    D = rng.choice([64, 128, 128, 72, 40, 104, 192, 256])
    hk = rng.choice([1, 2, 3, 8])
    group = rng.choice([1, 2, 3, 5, 8, 16])
    most = 3 if seed % 3 == 0 else log(1, 300)
    new = [rng.randint(0, most) for _ in range(seqs)]
    if sum(new) == 0:
        new[0] = 1
    while sum(new) * group * hk > 6000 and max(new) > 1:
        new = [n // 2 for n in new]
    new[0] = max(1, new[0])
    before = [rng.choice([0, rng.randint(0, 40), log(1, 900)]) for _ in range(seqs)]
    b = Batch(new, before, rng.choice([1, 8, 16, 24, 32, 48, 64, 128, 160, 256, 384]), hk * group, hk, D, dtype, seed=seed,
              spare=rng.randint(0, 40), heads_first=rng.random() < 0.5, pad=rng.choice([0, 0, 8, 1]))
    b.check(causal=rng.random() < 0.8, window=rng.choice([0, 0, 1, rng.randint(1, 400)]))


CHECKED = r"""
import torch
import paper_2605_07355_b200 as P
from tests.paged import ints
from tests.test_gpu_attend import Batch, CASES
assert P.LIB_PATH.endswith("libttf_b200_checked.so")
for case in CASES:
    *shape, mask = case
    Batch(*shape).check(**mask)                              # (ends with a clean status)
for new, before in (([1, 1], [300, 40]), ([150, 90], [200, 0]), ([130], [9000])):
    b = Batch(new, before, 16, 8, 2, 128)
    a = b.on_device()
    assert P.ttf_debug_set_check_slack(b.rows - sum(new) + 1) == 0      # the last row is out of bounds now: reported, left out
    out = P.ttf_attend(*a, b.scale, out=torch.full_like(a[0], 3))
    assert P.ttf_paged_status() == P.TTF_ERR_BOUNDS
    assert (out[sum(new) - 1] == 3).all()
    P.ttf_debug_set_check_slack(0)
    b.check()
k = torch.ones(5, 2, 64, device="cuda", dtype=torch.bfloat16)
kc, vc = (torch.zeros(2, 4, 2, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
P.ttf_debug_set_check_slack(1)                               # the last slot of the cache, the last heads of the rows
P.ttf_cache_append(k, k, kc, vc, ints([0, 5]), ints([8]), ints([[0, 1]]))
assert P.ttf_paged_status() == P.TTF_ERR_BOUNDS and (kc[1, 3] == 0).all()
P.ttf_debug_set_check_slack(0)
P.ttf_cache_append(k, k, kc, vc, ints([0, 5]), ints([8]), ints([[0, 1]]))
assert P.ttf_paged_status() == 0 and (kc[1, 3] == 1).all() and (vc[0, 3] == 1).all()
print("checked build ok")
"""


def test_checked_build():
    from paper_2605_07355_b200 import build
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, TTF_B200_LIB=build.build(checked=True))
    out = subprocess.run([sys.executable, "-c", CHECKED], env=env, cwd=root, capture_output=True, text=True, timeout=900)
    assert out.returncode == 0 and "checked build ok" in out.stdout, out.stdout[-2000:] + out.stderr[-4000:]


FIRST = """
import torch
import paper_2605_07355_b200 as P
from tests.test_gpu_attend import Batch
b = Batch({new}, [40, 300], 16, 8, 2, 128, "{dtype}")
q, k, v, st, ln, tb = b.on_device()
out, turned = torch.zeros_like(q), torch.zeros_like(q)
pos, freq = torch.arange(q.shape[0], device="cuda", dtype=torch.int32), torch.rand(64, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    P.ttf_rotate(q, None, pos, freq, out_q=turned)
    P.ttf_attend(q, k, v, st, ln, tb, b.scale, out=out)
g.replay()
assert P.ttf_paged_status() == 0
m = b.start[-1]
assert torch.equal(P.ttf_attend(q, k, v, st, ln, tb, b.scale)[:m], out[:m])
assert torch.equal(P.ttf_rotate(q, None, pos, freq)[0], turned)
"""


@pytest.mark.parametrize("new,dtype", [([1, 1], "bf16"), ([3, 200], "bf16"), ([1, 1], "f32"), ([3, 200], "f32")])
def test_a_process_may_begin_with_a_capture(new, dtype):
    r = subprocess.run([sys.executable, "-c", FIRST.format(new=new, dtype=dtype)], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_numbers_beyond_an_int_are_refused():
    q, out = torch.zeros((4, 2, 8), device="cuda"), torch.zeros((4, 2, 8), device="cuda")
    pos, freq = torch.zeros((4, 3), device="cuda", dtype=torch.int32), torch.ones(4, device="cuda")
    P.ttf_rotate(q, None, pos, freq, sections=(2, 1, 1), out_q=out)
    with pytest.raises((OverflowError, ValueError)):
        P.ttf_rotate(q, None, pos, freq, sections=(2**32 + 2, 1, 1), out_q=out)
    with pytest.raises((OverflowError, ValueError)):
        P.ttf_rotate(q, None, pos, freq, sections=(2, 1, 1), rot_dim=2**32 + 8, out_q=out)
    b = Batch([1], [3], 16, 2, 1, 8, "f32")
    q, k, v, st, ln, tb = b.on_device()
    with pytest.raises((OverflowError, ValueError)):
        P.ttf_attend(q, k, v, st, ln, tb, 1.0, window=2**32 + 1, out=torch.zeros_like(q))
