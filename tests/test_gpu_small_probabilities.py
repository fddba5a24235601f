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


def dominated(n, Hq, Hkv, h, gap, seed):
    """Queries, keys and values of n tokens: key 0 lies `gap` above the others for every query and has next to no value."""
    q, k, v = (rand(seed + i, n, m, h, dt=torch.float32) * s for i, (m, s) in enumerate(((Hq, 0.3), (Hkv, 0.3), (Hkv, 100.0))))
    q[:, :, 3] = 4.0
    k[:, :, 3] = 0.0
    k[0, :, 3] = gap * math.sqrt(h) / 4.0
    v[0] *= 2.0 ** -19
    return q.half(), k.half(), v.half()


def check_out(q, k, v, ctx, window, sinks, out):
    """out = P v: P is rounded once to 11 bits, its exponent is off by the score's 32-bit sum, the sum that it is divided by likewise, and the
    result is rounded once."""
    u, eps, (n, Hq, h), T = W.U[HF], W.EPS, q.shape, k.shape[0]
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    mask = W.seen(torch.arange(ctx, ctx + n), T, window, sinks)
    want, bound = torch.zeros_like(q), torch.zeros_like(q)
    for a in range(Hq):
        b = a // (Hq // k.shape[1])
        z = q[:, a] @ k[:, b].T / math.sqrt(h)
        p = torch.softmax(z.masked_fill(~mask, -math.inf), 1)
        assert float(p[mask].min()) > 2.0 ** -24 and (n < 100 or float(p[mask].median()) < 2.0 ** -19)
        e_s = ((h + 8) * 2.0 ** -24 / math.sqrt(h) * (q[:, a].abs() @ k[:, b].abs().T)).masked_fill(~mask, 0.0).amax(1)
        want[:, a] = p @ v[:, b]
        bound[:, a] = (p * (u + 2 * e_s + 2 * eps)[:, None]) @ v[:, b].abs()
    W.check("out", out, want, bound + u * (want.abs() + bound) + 2.0 ** -25)


@pytest.mark.parametrize("Hq, Hkv, h", [(2, 1, 64), (4, 4, 80), (4, 1, 128), (2, 2, 256), (8, 1, 32), (6, 2, 96)])
@pytest.mark.parametrize("window, sinks", [(0, 0), (100, 1)])
def test_outputs_beside_a_dominant_key(Hq, Hkv, h, window, sinks):
    n, scale = 600, 1 / math.sqrt(h)
    q, k, v = dominated(n, Hq, Hkv, h, 15.0, h)
    out, _ = R.rlgen_window_attention(q, k, v, i32([0, n]), n, window, sinks, scale)
    check_out(q, k, v, 0, window, sinks, out)


@pytest.mark.parametrize("Hq, Hkv, h", [(8, 2, 64), (4, 4, 80), (4, 1, 128), (2, 2, 256)])
@pytest.mark.parametrize("window, sinks", [(0, 0), (300, 1)])
@pytest.mark.parametrize("new", [1, 5, 200])
def test_outputs_over_pages_beside_a_dominant_key(Hq, Hkv, h, window, sinks, new):
    """Single tokens by the waves of several blocks and by one wave each, chunks whole and with their keys parted."""
    n, P, scale = 900, 16, 1 / math.sqrt(h)
    q, k, v = dominated(n, Hq, Hkv, h, 15.0, 100 + h)
    need = -(-n // P)
    ids = torch.randperm(need, generator=torch.Generator().manual_seed(h))
    pages = torch.zeros(need, 2, Hkv, P, h, dtype=HF, device="cuda")
    for e in range(need):
        part = torch.stack([k[e * P:(e + 1) * P], v[e * P:(e + 1) * P]]).transpose(1, 2)
        pages[int(ids[e]), :, :, :part.shape[2]] = part
    for S in (1, 2048 // Hkv) if new == 1 else (1,):
        table = ids.int().cuda().view(1, need).expand(S, need).contiguous()
        qs = q[n - new:].repeat(S, 1, 1)
        starts = torch.arange(S + 1, dtype=torch.int32, device="cuda") * new
        for ws in (None, torch.empty(16, dtype=torch.uint8, device="cuda")) if new > 1 else (None,):
            out, _ = R.rlgen_window_attention_paged(qs, pages, table, starts, i32([n] * S), new, n, window, sinks, scale, workspace=ws)
            check_out(q[n - new:], k, v, n - new, window, sinks, out[-new:])
