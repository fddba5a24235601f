"""Gradients where every row sees few keys: their dS nearly cancel, and a result that is rounded once must not be further off than that
rounding.  What else errs is 32-bit sums and dS kept to twice the type's bits, below a hundredth of it."""
import pytest
import torch

import window_reference as W
from test_gpu_operators import BF, HF, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("lens, Hq, Hkv, h, window, sinks", [
    ([2] * 20, 4, 4, 32, 0, 0), ([2, 1, 3] * 7, 12, 2, 96, 0, 0), ([64, 14, 5], 8, 2, 64, 0, 0), ([300, 120], 4, 2, 80, 25, 0), ([200], 4, 1, 128, 2, 0),
    ([40, 33], 2, 2, 256, 0, 0), ([90, 100], 8, 1, 128, 32, 0)])
def test_gradients_are_off_by_one_rounding(lens, Hq, Hkv, h, window, sinks, dt):
    q, k, v, st, out, lse, do, got = attend(lens, Hq, Hkv, h, window, sinks, dt, seed=len(lens) + h)
    want, at = {"dq": [], "dk": []}, 0
    for n in lens:
        part = slice(at, at + n)
        r = W.attention(q[part], k[part], v[part], 0, window, sinks, h ** -0.5, dt, do[part])
        for name in want:
            want[name].append(r[name][0])
        at += n
    for name, parts in want.items():
        exact = torch.cat(parts)
        once = float((exact.to(dt).double() - exact).norm())
        assert float((got[name].double().cpu() - exact).norm()) <= 1.1 * once, name
