"""The first calls of a process from several host threads at once: none of them may see a kernel whose launch limits (dynamic
shared memory, large clusters) another thread is still about to set."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

THREADS = """
import threading
import torch
import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import binding
from tests.test_gpu_attend import Batch
binding._marshal()
b = Batch({new}, {before}, 16, {heads}, 1, {D}, "{dtype}")
args = b.on_device()
n = 8
outs = [torch.zeros_like(args[0]) for _ in range(n)]
streams = [torch.cuda.Stream() for _ in range(n)]
torch.cuda.synchronize()
ready, failed = threading.Barrier(n), []

def first(i):
    torch.cuda.set_device(0)
    with torch.cuda.stream(streams[i]):
        ready.wait()
        try:
            P.ttf_attend(*args, b.scale, out=outs[i])
        except Exception as e:
            failed.append(repr(e))

threads = [threading.Thread(target=first, args=(i,)) for i in range(n)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert not failed, failed
assert P.ttf_paged_status() == 0
assert all(torch.equal(o, outs[0]) for o in outs) and bool((outs[0][0] != 0).any())
"""

# new, before, heads, D, dtype: clusters of 16 of the few-row kernels, shared memory beyond 48 KB of the others
CASES = [([1], [6000], 8, 128, "bf16"), ([1], [6000], 8, 256, "bf16"), ([1], [6000], 8, 128, "f32"), ([300], [10], 4, 128, "bf16"),
         ([300], [10], 4, 64, "f32")]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_threads_that_begin_together(case):
    new, before, heads, D, dtype = case
    code = THREADS.format(new=new, before=before, heads=heads, D=D, dtype=dtype)
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-500:] + r.stderr[-2000:]


CAPTURE = """
import torch
import paper_2605_07355_b200 as P
from tests.test_gpu_attend import Batch
b = Batch([1], [6000], 16, 8, 1, {D}, "{dtype}", spare=0)
args = b.on_device()
out = torch.zeros_like(args[0])
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    P.ttf_attend(*args, b.scale, out=out)
g.replay()
assert P.ttf_paged_status() == 0
assert torch.equal(P.ttf_attend(*args, b.scale, out=torch.zeros_like(out)), out) and bool((out != 0).any())
"""


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (256, "bf16"), (128, "f32"), (256, "f32")])
def test_a_capture_whose_clusters_the_device_is_asked_about(D, dtype):
    """the first call of a process, captured, with so long a sequence that sixteen CTAs may share it"""
    r = subprocess.run([sys.executable, "-c", CAPTURE.format(D=D, dtype=dtype)],
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-500:] + r.stderr[-2000:]
