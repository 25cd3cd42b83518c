"""No report is lost between a query that takes the status word and calls on other streams that report meanwhile."""
import threading

import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import binding as B
from tests.paged import ints
from tests.test_gpu_attend import Batch

pytestmark = pytest.mark.gpu


class Bad:
    """an append whose sequence is longer than its table: reported, nothing stored"""

    def __init__(self):
        self.k = torch.ones(1, 1, 32, device="cuda")
        self.cache = torch.zeros(1, 4, 1, 32, device="cuda")
        self.args = ints([0, 1]), ints([5]), ints([[0]])

    def call(self, stream):
        P.ttf_cache_append(self.k, self.k, self.cache, self.cache, *self.args, stream=stream)


def test_a_report_that_comes_while_another_is_taken():
    """The first call reports that a wait ran out, the second one, on another stream, that a length is out of bounds, at times
    spread around the query.  Whatever comes first, one of two queries tells the second report."""
    b = Batch([1, 1], [300, 40], 16, 8, 2, 128)
    args, bad, other = b.on_device(), Bad(), torch.cuda.Stream()
    out = torch.zeros_like(args[0])
    torch.cuda.synchronize()
    assert P.ttf_paged_status() == B.TTF_OK
    for i in range(200):
        P.ttf_debug_set_wait(32, 16)
        try:
            P.ttf_attend(*args, b.scale, out=out)
        finally:
            P.ttf_debug_set_wait()
        torch.cuda.current_stream().synchronize()
        with torch.cuda.stream(other):
            torch.cuda._sleep(500 * i)                      # up to some 50 us
        bad.call(other)
        first = P.ttf_paged_status()
        other.synchronize()
        second = P.ttf_paged_status()
        assert first != B.TTF_OK and B.TTF_ERR_BOUNDS in (first, second), (i, first, second)
        assert P.ttf_paged_status() == B.TTF_OK


def test_queries_of_several_threads():
    """every thread's report is told to somebody, and none is left behind"""
    bad, n, rounds = [Bad() for _ in range(4)], 4, 50
    streams = [torch.cuda.Stream() for _ in range(n)]
    torch.cuda.synchronize()
    assert P.ttf_paged_status() == B.TTF_OK
    told, failed, step = [], [], threading.Barrier(n)

    def work(i):
        try:
            torch.cuda.set_device(0)
            for _ in range(rounds):
                bad[i].call(streams[i])
                got = P.ttf_paged_status(streams[i])
                told.append(got)
                step.wait()                                 # all reports have been made and asked for
                if i == 0:
                    assert B.TTF_ERR_BOUNDS in told and set(told) <= {B.TTF_OK, B.TTF_ERR_BOUNDS}
                    told.clear()
                    assert P.ttf_paged_status(streams[i]) == B.TTF_OK
                step.wait()
        except BaseException as e:
            failed.append(repr(e))
            step.abort()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failed, failed
    assert P.ttf_paged_status() == B.TTF_OK


def test_a_query_beside_a_capture():
    """a query on one stream does not disturb the capture that another thread has open"""
    b = Batch([1], [40], 16, 8, 2, 128)
    args, out = b.on_device(), None
    out = torch.zeros_like(args[0])
    want = P.ttf_attend(*args, b.scale, out=torch.zeros_like(out))
    bad, other = Bad(), torch.cuda.Stream()
    bad.call(other)
    torch.cuda.synchronize()
    graph, got = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        P.ttf_attend(*args, b.scale, out=out)
        t = threading.Thread(target=lambda: (torch.cuda.set_device(0), got.append(P.ttf_paged_status(other))))
        t.start()
        t.join()
    graph.replay()
    torch.cuda.synchronize()
    assert got == [B.TTF_ERR_BOUNDS] and torch.equal(out, want) and P.ttf_paged_status() == B.TTF_OK
