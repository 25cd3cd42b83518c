"""Matching and attention on the tensor cores at the same time, both in clusters that hold tensor memory while they wait."""
import pytest
import torch

import paper_2605_07355_b200 as P
from tests.parity import to_device
from tests.test_gpu_attend import Batch
from tests.test_gpu_parity import corr_clip

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
def test_on_two_streams(D):
    clip = to_device(corr_clip(8, 16, 16, 1024, seed=7, dtype="bf16"))
    b = Batch([150, 90], [4000, 2600], 64, 4, 1, D)
    args = b.on_device()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [torch.zeros_like(args[0]) for _ in range(2)]
    clips = [P.ttf_compress(clip, 1, 0.7, stream=s) for s in streams[2:]]
    want = P.ttf_attend(*args, b.scale, out=torch.zeros_like(args[0]))
    torch.cuda.synchronize()
    n = int(clips[0][1])
    tokens = clips[0][0][:n].clone()
    torch.cuda.synchronize()
    for _ in range(200):
        for s, o in zip(streams[:2], outs):
            P.ttf_attend(*args, b.scale, out=o, stream=s)
        for s, c in zip(streams[2:], clips):
            P.ttf_compress(clip, 1, 0.7, *c, stream=s)
    torch.cuda.synchronize()
    assert P.ttf_paged_status() == 0 and all(torch.equal(o, want) for o in outs)
    for s, c in zip(streams[2:], clips):
        assert P.ttf_last_device_status(s) == 0 and int(c[1]) == n and torch.equal(c[0][:n], tokens)
