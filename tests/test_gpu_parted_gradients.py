"""Gradients of keys whose queries are parted over blocks (few kv heads, long sequences), against the plain 64-bit form
(window_reference) with the bounds that it derives from the types."""
import pytest
import torch

from test_gpu_operators import BF, HF, R, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens, Hq, Hkv, h, window, sinks", [
    ([700, 513], 8, 1, 64, 0, 0), ([1200], 12, 1, 96, 0, 0), ([0, 900, 1, 130], 5, 1, 80, 0, 0), ([1100], 4, 2, 128, 0, 0), ([1400], 8, 1, 32, 300, 0),
    ([1400, 40], 8, 1, 64, 600, 5), ([1300], 8, 1, 48, 900, 200), ([1500], 4, 1, 256, 0, 0), ([1300], 16, 2, 112, 40, 4), ([640], 40, 1, 16, 640, 0)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_gradients_of_few_long_sequences(lens, Hq, Hkv, h, window, sinks, dt):
    attend(lens, Hq, Hkv, h, window, sinks, dt, seed=sum(lens) + h)


def test_parted_gradients_are_the_same_every_time():
    q, k, v, st, out, lse, do, got = attend([900, 650], 8, 1, 64, 500, 3, BF)
    for _ in range(3):
        again = R.rlgen_window_attention_backward(q, k, v, out, lse, do, st, 900, 500, 3, 0.125)
        assert all(torch.equal(got[name], x) for name, x in zip(("dq", "dk", "dv"), again))
