"""One decoding sequence of some thousand slots: sixteen CTAs share it where the device can place such a cluster, eight where it
cannot; heads of every width."""
import pytest

from tests.test_gpu_attend import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype,page", [(64, "bf16", 16), (128, "bf16", 16), (128, "bf16", 7), (192, "bf16", 16), (192, "bf16", 24),
                                          (256, "bf16", 16), (256, "bf16", 5), (128, "f32", 16), (200, "f32", 16), (256, "f32", 16)])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (8, 2)])
def test_long_sequence_wide_heads(D, dtype, page, heads, kv_heads):
    Batch([1], [5000], page, heads, kv_heads, D, dtype).check()


@pytest.mark.parametrize("D,dtype", [(192, "bf16"), (256, "bf16"), (256, "f32")])
def test_window_and_two_sequences(D, dtype):
    Batch([1, 1], [5000, 17], 16, 2, 1, D, dtype).check()
    Batch([2], [6000], 16, 2, 1, D, dtype).check(window=4500)
