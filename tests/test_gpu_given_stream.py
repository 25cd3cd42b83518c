"""Outputs that the binding makes for a call on a given stream: their memory is not in use on the current stream any more, and is
not handed out again while the current stream still reads them."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.paged import ints
from tests.parity import to_device
from tests.test_gpu_attend import Batch
from tests.test_gpu_parity import corr_clip

pytestmark = pytest.mark.gpu

F, H, W, C = 6, 6, 7, 256


def calls():
    """name -> a function of the stream that returns the defined part of all outputs"""
    clip, other = (to_device(corr_clip(F, H, W, C, seed=s, dtype="bf16")) for s in (3, 4))
    n = {"clip": int(P.ttf_compress(clip, 1, 0.7)[1]), "other": int(P.ttf_compress(other, 1, 0.7)[1])}
    seg = int(P.ttf_compress_segment(clip, 1, 0.7, 1)[1])
    q = P.ttf_query(clip, 1, 0.7)
    tokens = P.ttf_compress(clip, 1, 0.7)[0][:n["clip"]].contiguous()
    b = Batch([1, 70], [300, 40], 16, 8, 2, 64, spare=0)
    bq, bk, bv, st, ln, tb = b.on_device()
    rows = bq.shape[0]
    k, v = torch.randn(rows, 2, 64, device="cuda").bfloat16(), torch.randn(rows, 2, 64, device="cuda").bfloat16()
    pos, freq = torch.arange(rows, dtype=torch.int32, device="cuda"), torch.rand(32, device="cuda")
    ck, cv = bk.clone(), bv.clone()
    torch.cuda.synchronize()                                # (the calls run on other streams than the one that makes the inputs)

    def cut(out, m):
        return [out[0][:m], out[1], out[2][:m]]

    def batch(stream):
        t, c, p = P.ttf_compress_batch([clip, other], 1, 0.7, stream=stream)
        return [t[0][:n["clip"]], t[1][:n["other"]], *c, p[0][:n["clip"]], p[1][:n["other"]]]

    return {
        "compress": lambda s: cut(P.ttf_compress(clip, 1, 0.7, stream=s), n["clip"]),
        "batch": batch,
        "mean": lambda s: cut(P.ttf_compress_mean(clip, 1, 0.7, stream=s), n["clip"]),
        "segment": lambda s: cut(P.ttf_compress_segment(clip, 1, 0.7, 1, stream=s), seg),
        "query": lambda s: list(P.ttf_query(clip, 1, 0.7, stream=s).values()),
        "restore": lambda s: list(P.ttf_restore(tokens, F, H, W, q["anchor"], q["keep"], q["dst"], stream=s)),
        "histogram": lambda s: [P.ttf_sim_histogram(q["best_sim"], q["anchor"], F, H, W, 64, stream=s)],
        "stats": lambda s: [P.ttf_stats(q["best_sim"], q["keep"], q["anchor"], F, H, W, 0.7, stream=s)],
        "rotate": lambda s: list(P.ttf_rotate(bq, k, pos, freq, stream=s)),
        "append": lambda s: [P.ttf_cache_append(k, v, ck, cv, st, ln, tb, pos, freq, q=bq, stream=s)],
        "attend": lambda s: [P.ttf_attend(bq, bk, bv, st, ln, tb, b.scale, stream=s)],
    }


NAMES = ["compress", "batch", "mean", "segment", "query", "restore", "histogram", "stats", "rotate", "append", "attend"]


def alone(f, stream):
    """the outputs of a call that has the GPU to itself (and the stream's own scratch is there after it)"""
    out = f(stream)
    torch.cuda.synchronize()                                # (the copies are made on the current stream)
    out = [t.clone() for t in out]
    torch.cuda.synchronize()
    return out


def whole(t):
    return torch.empty(t.untyped_storage().nbytes(), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("as_int", [False, True])
def test_memory_that_the_current_stream_still_writes(name, as_int):
    f, side = calls()[name], torch.cuda.Stream()
    given = side.cuda_stream if as_int else side
    want = alone(f, given)
    junk = [whole(t) for t in f(None)]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                           # some 10 ms, and then all of it is written
    for i in range(len(junk)):
        junk[i].fill_(0x55)
    del junk
    got = f(given)
    side.synchronize()
    torch.cuda.synchronize()
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_reads(name):
    f, side = calls()[name], torch.cuda.Stream()
    want = alone(f, side)
    got = f(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(20_000_000)
    copies = [t.clone() for t in got]                       # the current stream goes on with the outputs, and the caller drops them
    sizes = [t.untyped_storage().nbytes() for t in got]
    del got
    with torch.cuda.stream(side):
        for size in sizes:
            torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0x55)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies, want))


@pytest.mark.parametrize("legacy", [0, 1])
def test_the_default_stream_by_its_number(legacy):
    b = Batch([1, 70], [300, 40], 16, 8, 2, 64)
    args = b.on_device()
    m = b.start[-1]
    want = P.ttf_attend(*args, b.scale)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = P.ttf_attend(*args, b.scale, stream=legacy)
    torch.cuda.synchronize()
    assert torch.equal(got[:m], want[:m])


def test_a_given_stream_within_a_capture():
    """the output of a call on a stream that was forked within a capture belongs to the graph"""
    b = Batch([3], [60], 16, 8, 2, 64, spare=0)
    args = b.on_device()
    want = P.ttf_attend(*args, b.scale)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        out = P.ttf_attend(*args, b.scale, stream=side)
        here.wait_stream(side)
        twice = out + out
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(twice, want + want)
