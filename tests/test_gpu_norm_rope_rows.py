"""Norm and rotation, and their gradients, of more rows than a launch has blocks and waves: the walk from row to row, against the 64-bit
form; and the table of angles against numpy's."""
import numpy as np
import pytest
import torch

import window_reference as W
from test_gpu_operators import BF, HF, R, i32, rand, rope_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1500, 4096 + 5, 9001])
@pytest.mark.parametrize("Hq, Hkv, h, r, src, dt", [(4, 1, 64, 64, BF, BF), (3, 3, 80, 20, HF, HF), (2, 1, 128, 126, torch.float32, BF), (1, 1, 256, 0, torch.float32, HF)])
def test_many_rows(rows, Hq, Hkv, h, r, src, dt):
    rope, pos, qkv, gq, gk = rope_case(Hq, Hkv, h, r, rows, src, rows + h)
    gains = torch.cat([gq.expand(Hq, h), gk.expand(Hkv, h)])
    x = qkv.reshape(rows, Hq + 2 * Hkv, h)
    want, bound = W.norm_rope(x[:, : Hq + Hkv], None, 1e-5, rope, pos, gains, dt)
    q, k, v = R.rlgen_qk_norm_rope(qkv, gq, gk, 1e-5, rope, pos, n_kv_heads=Hkv, dtype=dt)
    W.check("q", q, want[:, :Hq], bound[:, :Hq])
    W.check("k", k, want[:, Hq:], bound[:, Hq:])
    assert torch.equal(v, x[:, Hq + Hkv:].to(dt))
    P, n_pages = 16, -(-rows // 16) + 3
    slots = torch.from_numpy(np.random.default_rng(rows).permutation(n_pages * P)[:rows].astype(np.int32))
    slots[::97] = -1
    pages = torch.full((n_pages, 2, Hkv, P, h), 7.0, dtype=dt, device="cuda")
    q2 = R.rlgen_qk_norm_rope(qkv, gq, gk, 1e-5, rope, pos, pages=pages, slots=slots.cuda())
    flat = torch.full((n_pages * P, 2, Hkv, h), 7.0, dtype=dt, device="cuda")
    on = (slots >= 0).cuda()
    flat[slots.cuda()[on].long()] = torch.stack([k[on], v[on]], 1)
    assert torch.equal(q2, q) and torch.equal(pages, flat.view(n_pages, P, 2, Hkv, h).permute(0, 2, 3, 1, 4))
    dq, dk, dv = (rand(rows + i, rows, n, h, dt=dt, scale=0.3) for i, n in enumerate((Hq, Hkv, Hkv)))
    dqkv, dgq, dgk = R.rlgen_qk_norm_rope_backward(qkv, gq, gk, 1e-5, rope, pos, dq, dk, dv)
    dx, b, dn, size = W.norm_rope_backward(x[:, : Hq + Hkv], torch.cat([dq, dk], 1), gains, 1e-5, rope, pos)
    got = dqkv.reshape(rows, -1, h)
    W.check("dqkv", got[:, : Hq + Hkv], dx, b + W.U[src] * (dx.abs() + b) + (2.0 ** -25 if src == HF else 0.0))
    assert torch.equal(got[:, Hq + Hkv:], dv.to(src))
    # (a lane adds up to 9001 / 1024 rows of all heads in turn, then blocks and runs: below 512 roundings)
    W.check("dq_gain", dgq, dn[:, :Hq].sum((0, 1)), 512 * 2.0 ** -22 * size[:, :Hq].sum((0, 1)))
    W.check("dk_gain", dgk, dn[:, Hq:].sum((0, 1)), 512 * 2.0 ** -22 * size[:, Hq:].sum((0, 1)))


@pytest.mark.parametrize("max_pos, r, theta", [(1, 2, 1e4), (777, 20, 1e4), (40000, 128, 5e5), (100, 256, 10.0)])
def test_the_table_of_angles(max_pos, r, theta):
    ang = np.arange(max_pos, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(r // 2) / r)[None, :]
    got = R.rlgen_rope_table(max_pos, r, theta).double().cpu().numpy()
    assert got.shape == (max_pos, r // 2, 2)
    # rounded once to 24 bits (2^-25 at most below 1), the angle's own rounding in 64 bits below that
    assert np.abs(got - np.stack([np.cos(ang), np.sin(ang)], -1)).max() <= 2.0 ** -24
