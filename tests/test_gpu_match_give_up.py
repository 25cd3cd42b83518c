"""Clips of so few channels that the tcgen05 matching kernel's producer is through before anybody's wait runs out: a CTA stays until
its copies have landed and its products have ended, so that the CTA after it finds shared and tensor memory to itself."""
import pytest
import torch

import paper_2605_07355_b200 as P
from paper_2605_07355_b200 import binding as B
from tests.parity import to_device
from tests.test_gpu_parity import corr_clip

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [64, 192, 256, 1024])
@pytest.mark.parametrize("r", [1, 2])
def test_waits_that_run_out_behind_the_producer(C, r):
    clip, other = (to_device(corr_clip(8, 12, 12, c, seed=s, dtype="bf16")) for c, s in ((C, 83), (512, 84)))
    st = torch.cuda.Stream()
    P.ttf_set_match_kernel(2)
    try:
        with torch.cuda.stream(st):
            want, after = P.ttf_query(clip, r, 0.7), P.ttf_query(other, r, 0.7)
            assert P.ttf_last_device_status(st) == B.TTF_OK
            for _ in range(10):
                P.ttf_debug_set_wait(32, 16)
                try:
                    P.ttf_query(clip, r, 0.7)
                finally:
                    P.ttf_debug_set_wait()
                got = P.ttf_query(other, r, 0.7)            # the next CTAs on the same SMs
                assert P.ttf_last_device_status(st) == B.TTF_OK
                for k in after:
                    assert torch.equal(got[k], after[k]), k
            P.ttf_debug_set_wait(32, 16)
            try:
                P.ttf_query(clip, r, 0.7)
                assert P.ttf_last_device_status(st) == B.TTF_ERR_TIMEOUT
            finally:
                P.ttf_debug_set_wait()
            got = P.ttf_query(clip, r, 0.7)
            assert P.ttf_last_device_status(st) == B.TTF_OK and all(torch.equal(got[k], want[k]) for k in want)
    finally:
        P.ttf_set_match_kernel(0)
