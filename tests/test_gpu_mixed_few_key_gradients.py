"""Short sequences beside longer ones: the precision of a sequence's gradients is its own, whatever else is in the call."""
import pytest
import torch

import window_reference as W
from test_gpu_operators import BF, HF, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("lens, Hq, Hkv, h, window, sinks", [
    ([2] * 20 + [65], 4, 4, 32, 0, 0), ([2, 1, 3, 700] * 5, 12, 2, 96, 0, 0), ([64, 14, 300, 5], 8, 2, 64, 0, 0), ([200] + [2] * 12, 4, 1, 128, 90, 4),
    ([40, 33, 130], 2, 2, 256, 0, 0), ([3] * 9 + [400], 4, 4, 80, 0, 0), ([2] * 9 + [1500], 8, 1, 64, 600, 5)])
def test_short_sequences_are_off_by_one_rounding_beside_long_ones(lens, Hq, Hkv, h, window, sinks, dt):
    q, k, v, st, out, lse, do, got = attend(lens, Hq, Hkv, h, window, sinks, dt, seed=len(lens) + h)
    want, rows, at = {"dq": [], "dk": []}, [], 0
    for n in lens:
        if n <= 64:
            part = slice(at, at + n)
            r = W.attention(q[part], k[part], v[part], 0, window, sinks, h ** -0.5, dt, do[part])
            rows += range(at, at + n)
            for name in want:
                want[name].append(r[name][0])
        at += n
    for name, parts in want.items():
        exact = torch.cat(parts)
        once = float((exact.to(dt).double() - exact).norm())
        assert float((got[name][rows].double().cpu() - exact).norm()) <= 1.1 * once, name
