"""Plain 64-bit forms of the operators over packed rows and pages, with bounds on what 32-bit sums and 16-bit operands may be off.

Every bound follows from the formula: u is the unit roundoff of the operands' type (an output is rounded once, and so are the
probabilities and dS for their second products), EPS one of the 32-bit sums and of exp.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}      # 2^-p with p significant bits
EPS = 2.0 ** -20
TINY16 = 2.0 ** -25          # half the smallest fp16 number: what fp16 may lose of a small probability


def seen(pos, T, window, sinks):
    """[len(pos), T]: does the query at pos see the key"""
    i, j = torch.as_tensor(pos)[:, None], torch.arange(T)[None, :]
    ok = j <= i
    if window:
        ok = ok & ((j > i - window) | (j < sinks))
    return ok


def attention(q, k, v, ctx, window, sinks, scale, dt, do=None):
    """One sequence in 64 bits: q [n, Hq, h] at positions ctx .., k, v [T, Hkv, h].  {name: (value, bound)}."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    n, Hq, h = q.shape
    T, Hkv, _ = k.shape
    u = U[dt]
    shape_kv = k.shape
    mask = seen(torch.arange(ctx, ctx + n), T, window, sinks)
    if T == 0:                # (no key: amax and the sums below have nothing to go over)
        k, v, mask, T = q.new_zeros(1, Hkv, h), q.new_zeros(1, Hkv, h), torch.zeros(n, 1, dtype=torch.bool), 1
    out, lse = torch.zeros_like(q), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    b_out, b_lse = torch.zeros_like(q), torch.zeros(n, Hq, dtype=torch.float64)
    g = {x: (torch.zeros_like(y), torch.zeros_like(y)) for x, y in (("dq", q), ("dk", k), ("dv", v))}
    if do is not None:
        do = do.double().cpu()
        peak = float(do.abs().max()) if do.numel() else 0.0
    for a in range(Hq):
        b = a // (Hq // Hkv)
        s = (q[:, a] @ k[:, b].T * scale).masked_fill(~mask, -math.inf)
        live = mask.any(1)
        m = torch.where(live, s.amax(1), torch.zeros(n, dtype=torch.float64))
        e = torch.exp(s - m[:, None])
        z = e.sum(1)
        p = e / torch.where(live, z, torch.ones_like(z))[:, None]
        lse[:, a] = torch.where(live, torch.log(z) + m, lse[:, a])
        out[:, a] = p @ v[:, b]
        # of a score: a 32-bit sum of h products, then its share of the exponent's rounding
        e_s = ((h + 8) * 2.0 ** -24 * abs(scale) * (q[:, a].abs() @ k[:, b].abs().T)).masked_fill(~mask, 0.0).amax(1)
        e_p = 2 * e_s + EPS
        b_lse[:, a] = e_s + EPS * (1 + lse[:, a].abs().masked_fill(~live, 0.0))
        small = TINY16 if dt == torch.float16 else 0.0
        pv, vsum = p @ v[:, b].abs(), mask.double() @ v[:, b].abs()
        b_out[:, a] = u * (out[:, a].abs() + pv) * (1 + u) + e_p[:, None] * pv + small * vsum + (2.0 ** -25 if dt == torch.float16 else 0)
        if do is None:
            continue
        dp = do[:, a] @ v[:, b].T
        delta = (p * dp).sum(1)
        ds = p * (dp - delta[:, None])
        ds_small = 2.0 ** -21 * peak if dt == torch.float16 else 0.0
        e_dp = (h + 8) * 2.0 ** -24 * (do[:, a].abs() @ v[:, b].abs().T)
        e_delta = (do[:, a].abs() * b_out[:, a]).sum(1) + EPS * (do[:, a].abs() * out[:, a].abs()).sum(1)
        b_ds = (u + 2 * e_p[:, None] + EPS) * ds.abs() + p * (e_dp + e_delta[:, None]) * (1 + u) + ds_small * mask
        b_p = (u + e_p)[:, None] * p + small * mask
        for x, val, bound in (("dq", ds @ k[:, b] * scale, b_ds @ k[:, b].abs() * abs(scale)),):
            g[x][0][:, a] = val
            g[x][1][:, a] = bound + u * (val.abs() + bound) + 1e-7 * (ds.abs() @ k[:, b].abs()) + (2.0 ** -25 if dt == torch.float16 else 0)
        g["dk"][0][:, b] += ds.T @ q[:, a] * scale
        g["dk"][1][:, b] += b_ds.T @ q[:, a].abs() * abs(scale) + EPS * (ds.abs().T @ q[:, a].abs())
        g["dv"][0][:, b] += p.T @ do[:, a]
        g["dv"][1][:, b] += b_p.T @ do[:, a].abs() + EPS * (p.T @ do[:, a].abs())
    r = {"out": (out, b_out), "lse": (lse, b_lse)}
    if do is not None:
        for x in ("dk", "dv"):
            val, bound = g[x]
            g[x] = tuple(t[: shape_kv[0]] for t in (val, bound + u * (val.abs() + bound) + (2.0 ** -25 if dt == torch.float16 else 0)))
        r.update(g)
    return r


def check(name, got, want, bound):
    got = got.double().cpu()
    same = torch.isinf(want) & (got == want)
    far = torch.where(same, torch.zeros_like(got), (got - torch.where(same, got, want)).abs())
    ratio = far / torch.clamp(bound, min=1e-30)
    ratio = torch.where(far == 0, torch.zeros_like(ratio), ratio)
    worst = float(ratio.max()) if ratio.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3f} times its bound"      # (a NaN fails)
    return worst


def norm_rope(x, gain, eps, rope, positions, heads_gain, dt):
    """x [rows, heads, h] in 64 bits -> (value, bound) of the normalised and rotated heads; heads_gain [heads, h]."""
    x, rope = x.double().cpu(), None if rope is None else rope.double().cpu()
    r = 0 if rope is None else 2 * rope.shape[1]
    y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * heads_gain.double().cpu()
    out, size = y.clone(), y.abs()
    if r:
        c, s = rope[positions.long().cpu()][:, None, :, 0], rope[positions.long().cpu()][:, None, :, 1]
        a, b = y[..., : r // 2], y[..., r // 2: r]
        out[..., : r // 2], out[..., r // 2: r] = a * c - b * s, b * c + a * s
        both = a.abs() + b.abs()
        size = torch.cat([both, both, y[..., r:].abs()], -1)
    return out, U[dt] * out.abs() + EPS * size + (2.0 ** -25 if dt == torch.float16 else 0)


def norm_rope_backward(x, d, gain, eps, rope, positions):
    """Gradients in 64 bits: dx, its bound without the last rounding, and dy n per head (whose sums are the gains' gradients)."""
    x, d, gain = x.double().cpu(), d.double().cpu(), gain.double().cpu()
    h = x.shape[-1]
    dy, size = d.clone(), d.abs()
    if rope is not None:
        rope = rope.double().cpu()
        r = 2 * rope.shape[1]
        c, s = rope[positions.long().cpu()][:, None, :, 0], rope[positions.long().cpu()][:, None, :, 1]
        a, b = d[..., : r // 2], d[..., r // 2: r]
        dy[..., : r // 2], dy[..., r // 2: r] = a * c + b * s, b * c - a * s
        both = a.abs() + b.abs()
        size = torch.cat([both, both, d[..., r:].abs()], -1)
    inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x * inv
    t = dy * gain
    dx = inv * (t - n * (t * n).mean(-1, keepdim=True))
    st = size * gain.abs()
    return dx, 2 * EPS * inv * (st + n.abs() * (st * n.abs()).mean(-1, keepdim=True)), dy * n, size * n.abs()


def plan(ctx, new, P, free, head, table, max_rows):
    """Integers of the plan, sequence by sequence; table is changed in place."""
    total, starts, slots, pos = [], [0], [-1] * max_rows, [0] * max_rows
    at, faults, width = head, 0, len(table[0])
    for s, (c, n) in enumerate(zip(ctx, new)):
        if c < 0 or n < 0:
            faults |= 8
        c, n = max(c, 0), max(n, 0)
        had, need = -(-c // P), -(-(c + n) // P)
        if need > width:
            faults |= 4
        fresh = {}
        for e in range(had, need):
            fresh[e] = free[at] if at < len(free) else -1
            at += 1
            if e < width:
                table[s][e] = fresh[e]
        for i in range(n):
            r, p = starts[-1] + i, c + i
            page = fresh.get(p // P, table[s][p // P] if p // P < width else -1) if p // P < width else -1
            if r < max_rows:
                slots[r], pos[r] = (page * P + p % P if page >= 0 else -1), p
        total.append(c + n)
        starts.append(starts[-1] + n)
    if at > len(free):
        faults |= 2
    if starts[-1] > max_rows:
        faults |= 1
    return total, starts, slots, pos, [starts[-1], min(at, len(free)), max(total), faults]
