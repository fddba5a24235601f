"""fp16: what dv gets from small probabilities.  A key that takes nearly all of every row's mass leaves the others probabilities near 1e-6, below
the type's normal numbers; dv of those keys keeps the precision of one rounding all the same."""
import math

import pytest
import torch

import window_reference as W
from test_gpu_operators import HF, R, i32, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq, Hkv, h, n, window, sinks, gap", [
    (2, 1, 64, 600, 0, 0, 13.0), (4, 4, 80, 300, 0, 0, 14.0), (4, 1, 128, 500, 100, 1, 14.0), (2, 2, 256, 300, 0, 0, 13.0), (8, 1, 32, 1400, 200, 3, 12.0),
    (4, 2, 96, 60, 0, 0, 14.0)])
def test_values_gradients_beside_a_dominant_key(Hq, Hkv, h, n, window, sinks, gap):
    scale, dim = 1 / math.sqrt(h), 3
    q, k, v = (rand(h + i, n, m, h, dt=torch.float32) * 0.3 for i, m in enumerate((Hq, Hkv, Hkv)))
    q[:, :, dim] = 4.0
    k[:, :, dim] = 0.0
    k[0, :, dim] = gap / (4.0 * scale)                    # key 0 lies `gap` above the others for every query
    q, k, v = q.half(), k.half(), v.half()
    do = (rand(9, n, Hq, h, dt=torch.float32) * 500.0).half()
    st = i32([0, n])
    out, lse = R.rlgen_window_attention(q, k, v, st, n, window, sinks, scale)
    dv = R.rlgen_window_attention_backward(q, k, v, out, lse, do, st, n, window, sinks, scale)[2].double().cpu()
    # dv = P^T dout: P is rounded once to 11 bits (it stays above 2^-28), its exponent is off by the score's 32-bit sum, the result is rounded once
    u, eps = W.U[HF], W.EPS
    qd, kd, d = q.double().cpu(), k.double().cpu(), do.double().cpu()
    mask = W.seen(torch.arange(n), n, window, sinks)
    want, bound = torch.zeros_like(dv), torch.zeros_like(dv)
    for a in range(Hq):
        b = a // (Hq // Hkv)
        p = torch.softmax((qd[:, a] @ kd[:, b].T * scale).masked_fill(~mask, -math.inf), 1)
        assert float(p[mask].min()) > 2.0 ** -28 and float(p[mask].median()) < 2.0 ** -14
        e_s = ((h + 8) * 2.0 ** -24 * scale * (qd[:, a].abs() @ kd[:, b].abs().T)).masked_fill(~mask, 0.0).amax(1)
        want[:, b] += p.T @ d[:, a]
        bound[:, b] += (p * (u + 2 * e_s + 2 * eps)[:, None]).T @ d[:, a].abs()
    bound += u * (want.abs() + bound) + 2.0 ** -25
    past = want.to(HF).isinf()                            # (the dominant key's sum passes the type's largest number: its cast is an infinity)
    want[past] = want[past].sign() * math.inf
    W.check("dv", dv, want, bound)
