"""The operators over pages and packed rows against their plain 64-bit forms (window_reference), whose bounds are derived from the
types, at the sizes, masks and strides where they can go wrong."""
import math
import random

import numpy as np
import pytest
import torch

import window_reference as W

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def rand(seed, *shape, dt=BF, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dt).cuda()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts_of(lens):
    return i32([0] + list(np.cumsum(lens)))


# ------------------------------------------------------------------ plan


def run_plan(ctx, new, P, free, table, max_rows, head=None):
    t = i32(table)
    got = R.rlgen_plan_pages(i32(ctx), i32(new), P, i32(free), t, max_rows, None if head is None else i32([head]))
    want_table = [list(r) for r in table]
    want = W.plan(ctx, new, P, free, head or 0, want_table, max_rows)
    for name, g, w in zip(got._fields, got, want):
        assert g.tolist() == w, name
    assert t.tolist() == want_table
    return got, t


def tables(rng, ctx, new, P, spare=3):
    pages = list(range(sum(-(-(c + n) // P) for c, n in zip(ctx, new)) + spare))
    rng.shuffle(pages)
    width = max(1, max(-(-(c + n) // P) for c, n in zip(ctx, new)))
    table, at = [], 0
    for c in ctx:
        had = -(-c // P)
        table.append(pages[at:at + had] + [-7] * (width - had))
        at += had
    return table, pages[at:]


@pytest.mark.parametrize("S, P, hi, add", [(1, 8, 0, 1), (1, 16, 5, 3000), (3, 64, 100, 1), (64, 16, 40, 70), (255, 8, 30, 2), (257, 32, 200, 33),
                                           (1000, 16, 60, 1), (1100, 1024, 3000, 20), (5000, 8, 20, 3)])
def test_plan_matches_the_sequential_form(S, P, hi, add):
    rng = random.Random(S * 31 + P)
    ctx, new = [rng.randint(0, hi) for _ in range(S)], [rng.choice([0, 1, add, rng.randint(0, add)]) for _ in range(S)]
    table, free = tables(rng, ctx, new, P)
    run_plan(ctx, new, P, free, table, sum(new))
    run_plan(ctx, new, P, free, table, sum(new) + 37)          # rows that no sequence has
    run_plan(ctx, new, P, [9] * 5 + free, table, sum(new), head=5)


def test_plan_without_any_row():
    run_plan([0, 5, 8], [0, 0, 0], 8, [1, 2], [[-7, -7], [3, -7], [4, -7]], 0)
    run_plan([0], [0], 8, [], [[-7]], 4)


def test_plan_reports_what_does_not_fit():
    # rows beyond max_rows, an empty free list, a short table row, a negative length: each alone and together
    run_plan([0, 0], [9, 9], 8, [1, 2, 3, 4], [[-7] * 2] * 2, 11)
    run_plan([0, 3], [9, 9], 8, [1, 2], [[-7] * 2, [5, -7]], 18)
    run_plan([0, 3], [20, 9], 8, [1, 2, 3, 4, 6, 7], [[-7] * 2, [5, -7]], 29)
    run_plan([-4, 3], [9, -2], 8, [1, 2, 3], [[-7] * 2, [5, -7]], 9)
    run_plan([-4, 30], [40, 9], 8, [1, 2], [[-7] * 2, [5, 6]], 20)


def test_plans_follow_each_other_on_the_device():
    """Steps chained by the counts of the one before, without the host: as a whole pass in one."""
    rng = random.Random(3)
    S, P = 70, 16
    ctx, steps = [rng.randint(0, 50) for _ in range(S)], 20
    table, free = tables(rng, ctx, [steps] * S, P)
    t, lens, f, head = i32(table), i32(ctx), i32(free), None
    for _ in range(steps):
        plan = R.rlgen_plan_pages(lens, torch.ones_like(lens), P, f, t, S, head)
        lens, head = plan.total_lens, plan.counts[1:2]
    assert int(plan.counts[3]) == 0 and lens.tolist() == [c + steps for c in ctx]
    used = [row[: -(-(c + steps) // P)] for row, c in zip(t.tolist(), ctx)]
    flat = [p for row in used for p in row]
    assert len(set(flat)) == len(flat) and min(flat) >= 0


# ------------------------------------------------------------------ norm and rotation

SHAPES = [(4, 4, 32, 8), (8, 2, 64, 64), (32, 32, 80, 20), (5, 5, 96, 96), (6, 2, 112, 28), (32, 8, 128, 128), (3, 1, 16, 2), (8, 8, 256, 64), (2, 1, 208, 0),
          (7, 7, 48, 46)]


def rope_case(Hq, Hkv, h, r, rows, src, seed):
    rope = R.rlgen_rope_table(500, r, 1e4) if r else None
    rng = np.random.default_rng(seed)
    pos = i32(rng.integers(0, 500, size=rows).tolist())
    width = (Hq + 2 * Hkv) * h
    wide = rand(seed, rows, width + 24, dt=src, scale=2.0)
    qkv = wide[:, 8: 8 + width] if src != torch.float32 else wide[:, 4: 4 + width]
    gq, gk = (1 + rand(seed + i, h, dt=torch.float32, scale=0.2) for i in (1, 2))
    return rope, pos, qkv, gq, gk


@pytest.mark.parametrize("Hq, Hkv, h, r", SHAPES)
@pytest.mark.parametrize("src, dt", [(BF, BF), (HF, HF), (torch.float32, BF), (torch.float32, HF), (BF, HF), (HF, BF)])
def test_norm_rope_and_its_gradients(Hq, Hkv, h, r, src, dt):
    for rows in (1, 3, 37):
        rope, pos, qkv, gq, gk = rope_case(Hq, Hkv, h, r, rows, src, rows * 7 + h)
        gains = torch.cat([gq.expand(Hq, h), gk.expand(Hkv, h)])
        x = qkv.reshape(rows, Hq + 2 * Hkv, h)
        want, bound = W.norm_rope(x[:, : Hq + Hkv], None, 1e-5, rope, pos, gains, dt)
        q, k, v = R.rlgen_qk_norm_rope(qkv, gq, gk, 1e-5, rope, pos, n_kv_heads=Hkv, dtype=dt)
        W.check("q", q, want[:, :Hq], bound[:, :Hq])
        W.check("k", k, want[:, Hq:], bound[:, Hq:])
        assert torch.equal(v, x[:, Hq + Hkv:].to(dt))
        # into pages: one slot is outside, one row has none
        P, n_pages = 8, rows + 2
        pages = torch.full((n_pages, 2, Hkv, P, h), 7.0, dtype=dt, device="cuda")
        perm = np.random.default_rng(rows).permutation(n_pages * P)[:rows]
        slots = perm.copy()
        if rows == 37:
            slots[5], slots[11] = -1, n_pages * P
        q2 = R.rlgen_qk_norm_rope(qkv, gq, gk, 1e-5, rope, pos, pages=pages, slots=i32(slots.tolist()))
        assert torch.equal(q2, q)
        expect = torch.full_like(pages, 7.0)
        for i, s in enumerate(slots):
            if 0 <= s < n_pages * P:
                expect[s // P, 0, :, s % P], expect[s // P, 1, :, s % P] = k[i], v[i]
        assert torch.equal(pages, expect)
        # gradients
        dq, dk, dv = (rand(rows + i, rows, n, h + 8, dt=dt, scale=0.3)[:, :, :h].contiguous() for i, n in enumerate((Hq, Hkv, Hkv)))
        dqkv, dgq, dgk = R.rlgen_qk_norm_rope_backward(qkv, gq, gk, 1e-5, rope, pos, dq, dk, dv)
        dx, b, dn, size = W.norm_rope_backward(x[:, : Hq + Hkv], torch.cat([dq, dk], 1), gains, 1e-5, rope, pos)
        got = dqkv.reshape(rows, -1, h)
        small = 2.0 ** -25 if src == HF else 0.0
        W.check("dqkv", got[:, : Hq + Hkv], dx, b + W.U[src] * (dx.abs() + b) + small)
        assert torch.equal(got[:, Hq + Hkv:], dv.to(src))
        for name, g, part in (("dq_gain", dgq, slice(0, Hq)), ("dk_gain", dgk, slice(Hq, Hq + Hkv))):
            n = rows * (part.stop - part.start)
            W.check(name, g, dn[:, part].sum((0, 1)), (n + 64) * 2.0 ** -22 * size[:, part].sum((0, 1)))


def test_norm_rope_gradient_against_differences():
    """Along random directions the gradients are the change of the 64-bit form's weighted sum."""
    Hq, Hkv, h, r, rows = 4, 2, 48, 20, 9
    rope, pos, qkv, gq, gk = rope_case(Hq, Hkv, h, r, rows, torch.float32, 5)
    dq, dk, dv = (rand(60 + i, rows, n, h, dt=BF) for i, n in enumerate((Hq, Hkv, Hkv)))
    dqkv, dgq, dgk = R.rlgen_qk_norm_rope_backward(qkv, gq, gk, 1e-5, rope, pos, dq, dk, dv)
    x, weight = qkv.reshape(rows, -1, h).double().cpu(), torch.cat([dq, dk], 1).double().cpu()

    def value(x, gq, gk):
        gains = torch.cat([gq.expand(Hq, h), gk.expand(Hkv, h)])
        return float((W.norm_rope(x[:, : Hq + Hkv], None, 1e-5, rope, pos, gains, BF)[0] * weight).sum() + (x[:, Hq + Hkv:] * dv.double().cpu()).sum())

    g = torch.Generator().manual_seed(1)
    ex, eq, ek = (torch.randn(s, generator=g, dtype=torch.float64) for s in (x.shape, (h,), (h,)))
    t = 1e-5
    a, b = gq.double().cpu(), gk.double().cpu()
    slope = (value(x + t * ex, a + t * eq, b + t * ek) - value(x - t * ex, a - t * eq, b - t * ek)) / (2 * t)
    parts = [(dqkv.reshape(rows, -1, h).double().cpu(), ex), (dgq.double().cpu(), eq), (dgk.double().cpu(), ek)]
    got = sum(float((d * e).sum()) for d, e in parts)
    assert abs(got - slope) <= 1e-5 * sum(float((d * e).abs().sum()) for d, e in parts)


def test_gain_gradients_of_many_rows_are_the_same_every_time():
    Hq, Hkv, h, r, rows = 8, 2, 64, 64, 4100
    rope, pos, qkv, gq, gk = rope_case(Hq, Hkv, h, r, rows, BF, 11)
    dq, dk, dv = (rand(70 + i, rows, n, h, dt=BF) for i, n in enumerate((Hq, Hkv, Hkv)))
    first = R.rlgen_qk_norm_rope_backward(qkv, gq, gk, 1e-5, rope, pos, dq, dk, dv)
    gains = torch.cat([gq.expand(Hq, h), gk.expand(Hkv, h)])
    _, _, dn, size = W.norm_rope_backward(qkv.reshape(rows, -1, h)[:, : Hq + Hkv], torch.cat([dq, dk], 1), gains, 1e-5, rope, pos)
    W.check("dq_gain", first[1], dn[:, :Hq].sum((0, 1)), 512 * 2.0 ** -22 * size[:, :Hq].sum((0, 1)))
    for _ in range(3):
        again = R.rlgen_qk_norm_rope_backward(qkv, gq, gk, 1e-5, rope, pos, dq, dk, dv)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


# ------------------------------------------------------------------ attention over packed rows


def attend(lens, Hq, Hkv, h, window, sinks, dt, seed=0, grads=True, scale=None, amp=1.0):
    rows = sum(lens)
    scale = 1 / math.sqrt(h) if scale is None else scale
    fused = rand(seed, rows, (Hq + 2 * Hkv) * h, dt=dt, scale=amp)
    q, k, v = (x.view(rows, -1, h) for x in torch.split(fused, [Hq * h, Hkv * h, Hkv * h], 1))      # strided rows
    st = starts_of(lens)
    out, lse = R.rlgen_window_attention(q, k, v, st, max(lens + [1]), window, sinks, scale)
    do = rand(seed + 1, rows, Hq, h, dt=dt)
    got = {"out": out, "lse": lse}
    if grads:
        got.update(zip(("dq", "dk", "dv"), R.rlgen_window_attention_backward(q, k, v, out, lse, do, st, max(lens + [1]), window, sinks, scale)))
    at = 0
    for i, n in enumerate(lens):
        part = slice(at, at + n)
        want = W.attention(q[part], k[part], v[part], 0, window, sinks, scale, dt, do[part] if grads else None)
        for name, g in got.items():
            W.check(f"{name} of sequence {i} ({n} tokens)", g[part], *want[name])
        at += n
    return q, k, v, st, out, lse, do, got


@pytest.mark.parametrize("Hq, Hkv, h", [(4, 4, 32), (2, 1, 16), (8, 2, 64), (4, 4, 80), (3, 1, 80), (6, 2, 96), (2, 2, 48), (4, 1, 128), (5, 5, 112), (4, 2, 256), (2, 1, 208)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_attention_of_every_head_size(Hq, Hkv, h, dt):
    attend([1, 70, 0, 33, 131], Hq, Hkv, h, 0, 0, dt, seed=h)
    attend([65, 2, 200], Hq, Hkv, h, 37, 3, dt, seed=h + 1)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (7, 0), (31, 2), (32, 32), (64, 5), (65, 64), (100, 130), (127, 1), (128, 0), (500, 4), (2, 300)])
def test_attention_windows_and_sinks(window, sinks):
    attend([1, 2, 63, 64, 65, 129, 300, 457], 6, 2, 64, window, sinks, BF, seed=window)


@pytest.mark.parametrize("n, window, sinks", [(1500, 40, 4), (2600, 300, 130), (1290, 1, 1), (3000, 1000, 200)])
def test_gradients_of_sinks_that_later_queries_see_are_parted(n, window, sinks):
    """Sequences long enough that the queries beyond the window are added up in several parts, beside shorter ones that have fewer or none."""
    attend([n, n // 3, 20, n // 2 + 1], 2, 1, 32, window, sinks, BF, seed=n)
    attend([n], 3, 1, 16, window, sinks, HF, seed=n + 1)


@pytest.mark.parametrize("amp, scale", [(8.0, None), (0.01, None), (3.0, 0.0), (2.0, -0.2)])
def test_attention_of_peaked_flat_and_unusual_scores(amp, scale):
    """fp16 stays in its range: scores of hundreds, all alike, scale zero, scale below zero."""
    attend([90, 33], 4, 2, 64, 50, 2, HF, seed=5, amp=amp, scale=scale)
    attend([90, 33], 4, 2, 64, 0, 0, BF, seed=6, amp=amp, scale=scale)


@pytest.mark.parametrize("size", [2.0 ** -18, 2.0 ** 9])
def test_small_and_large_fp16_gradients_keep_their_precision(size):
    lens, Hq, Hkv, h, scale = [150], 2, 1, 64, 0.125
    q, k, v = (rand(i, 150, n, h, dt=HF) for i, n in enumerate((Hq, Hkv, Hkv)))
    st, do = starts_of(lens), (rand(9, 150, Hq, h, dt=torch.float32) * size).half()
    out, lse = R.rlgen_window_attention(q, k, v, st, 150, 0, 0, scale)
    got = R.rlgen_window_attention_backward(q, k, v, out, lse, do, st, 150, 0, 0, scale)
    want = W.attention(q, k, v, 0, 0, 0, scale, HF, do)
    for name, g in zip(("dq", "dk", "dv"), got):
        W.check(name, g, *want[name])


def test_attention_gradient_against_differences():
    lens, Hq, Hkv, h, window, sinks, scale = [40, 75], 4, 2, 32, 20, 3, 0.2
    q, k, v, st, out, lse, do, got = attend(lens, Hq, Hkv, h, window, sinks, HF, seed=21, scale=scale)
    x = [t.double().cpu() for t in (q, k, v)]
    g = torch.Generator().manual_seed(2)
    e = [torch.randn(t.shape, generator=g, dtype=torch.float64) for t in x]

    def value(t):
        s, at = 0.0, 0
        for n in lens:
            p = [(a + t * b)[at:at + n] for a, b in zip(x, e)]
            s += float((W.attention(*p, 0, window, sinks, scale, HF)["out"][0] * do[at:at + n].double().cpu()).sum())
            at += n
        return s

    slope = (value(1e-5) - value(-1e-5)) / 2e-5
    grads = [got[n].double().cpu() for n in ("dq", "dk", "dv")]
    allowed, at = 0.0, 0
    for n in lens:
        part = slice(at, at + n)
        want = W.attention(*(t[part] for t in x), 0, window, sinks, scale, HF, do[part])
        allowed += sum(float((want[name][1] * d[part].abs()).sum()) for name, d in zip(("dq", "dk", "dv"), e))
        at += n
    assert abs(sum(float((a * b).sum()) for a, b in zip(grads, e)) - slope) <= allowed + 1e-6 * abs(slope)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_a_query_does_not_see_never_reaches_it(bad):
    """An infinite or NaN key or value changes nothing for the queries that do not see it, in the same tile or not."""
    lens, Hq, Hkv, h, window, sinks, scale = [150, 60], 4, 2, 64, 33, 2, 0.125
    q, k, v = (rand(i, 210, n, h, dt=BF) for i, n in enumerate((Hq, Hkv, Hkv)))
    st = starts_of(lens)
    clean, clean_lse = R.rlgen_window_attention(q, k, v, st, 150, window, sinks, scale)
    for which, j in ((0, 70), (1, 70), (1, 0), (1, 149), (0, 149)):
        k2, v2 = k.clone(), v.clone()
        (k2, v2)[which][j, 1, 5] = bad
        out, lse = R.rlgen_window_attention(q, k2, v2, st, 150, window, sinks, scale)
        sees = torch.zeros(210, dtype=torch.bool)
        sees[:150] = W.seen(torch.arange(150), 150, window, sinks)[:, j]
        hit = torch.zeros(210, Hq, dtype=torch.bool)
        hit[:, 2:] = sees[:, None]                     # the query heads of kv head 1
        hit = hit.cuda()
        assert torch.isfinite(out[~hit]).all() and torch.isfinite(lse[~hit]).all()
        want = W.attention(q[:150], k[:150], v[:150], 0, window, sinks, scale, BF)
        far = (out[:150].double().cpu() - want["out"][0]).abs() <= want["out"][1]
        assert far[~hit[:150].cpu()].all()
        assert torch.equal(out[150:], clean[150:]) and torch.equal(lse[150:], clean_lse[150:])
        if which == 1:
            assert not torch.isfinite(out[hit][:, 5]).any() and torch.isfinite(out[hit][:, :5]).all()


def test_a_sequence_of_nan_leaves_the_others_gradients_alone():
    lens = [100, 77, 130]
    q, k, v, st, out, lse, do, got = attend(lens, 4, 2, 64, 40, 4, BF, seed=31)
    q, k, v, do = q.clone(), k.clone(), v.clone(), do.clone()
    for t in (q, k, v, do):
        t[100:177] = math.nan
    out2, lse2 = R.rlgen_window_attention(q, k, v, st, 130, 40, 4, 1 / 8)
    grads = R.rlgen_window_attention_backward(q, k, v, out2, lse2, do, st, 130, 40, 4, 1 / 8)
    for name, g in zip(("out", "lse", "dq", "dk", "dv"), (out2, lse2, *grads)):
        assert torch.equal(g[:100], got[name][:100]) and torch.equal(g[177:], got[name][177:]), name


def test_attention_returns_the_same_bits_every_time_and_on_any_stream():
    lens = [1, 700, 64, 333]
    q, k, v, st, out, lse, do, got = attend(lens, 8, 2, 128, 100, 4, BF, seed=41)
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            for _ in range(3):
                o, l = R.rlgen_window_attention(q, k, v, st, 700, 100, 4, 1 / math.sqrt(128))
                g = R.rlgen_window_attention_backward(q, k, v, o, l, do, st, 700, 100, 4, 1 / math.sqrt(128))
                torch.cuda.current_stream().synchronize()
                assert torch.equal(o, out) and torch.equal(l, lse)
                assert all(torch.equal(a, got[n]) for a, n in zip(g, ("dq", "dk", "dv")))


# ------------------------------------------------------------------ attention over pages


def cache(rng, totals, P, Hkv, h, dt, seed, spare=4):
    """Pages that hold NaN wherever no token of a sequence lies, the table, and the tokens' keys and values."""
    n_pages = sum(-(-t // P) for t in totals) + spare
    ids = list(range(n_pages))
    rng.shuffle(ids)
    pages = torch.full((n_pages, 2, Hkv, P, h), math.nan, dtype=dt, device="cuda")
    width = max(1, max(-(-t // P) for t in totals)) + 1
    table, kv, at = [], [], 0
    for i, t in enumerate(totals):
        need = -(-t // P)
        mine = ids[at:at + need]
        at += need
        table.append(mine + [-1] * (width - need))
        x = rand(seed + i, 2, t, Hkv, h, dt=dt)
        kv.append(x)
        for e, p in enumerate(mine):
            part = x[:, e * P:(e + 1) * P].transpose(1, 2)
            pages[p, :, :, :part.shape[2]] = part
    return pages, i32(table), kv


def attend_paged(totals, news, Hq, Hkv, h, P, window, sinks, dt, seed=0):
    pages, table, kv = cache(random.Random(seed), totals, P, Hkv, h, dt, seed)
    rows = sum(news)
    wide = rand(seed + 99, rows, Hq * h + 16, dt=dt)
    q = wide[:, 8:8 + Hq * h].view(rows, Hq, h) if rows > 1 else wide[:, 8:8 + Hq * h].reshape(rows, Hq, h)
    scale = 1 / math.sqrt(h)
    out, lse = R.rlgen_window_attention_paged(q, pages, table, starts_of(news), i32(totals), max(news), max(totals + [1]), window, sinks, scale)
    at = 0
    for i, (t, n) in enumerate(zip(totals, news)):
        want = W.attention(q[at:at + n], kv[i][0], kv[i][1], t - n, window, sinks, scale, dt)
        W.check(f"out of sequence {i} ({t} tokens)", out[at:at + n], *want["out"])
        W.check(f"lse of sequence {i} ({t} tokens)", lse[at:at + n], *want["lse"])
        at += n


HEADS = [(4, 4, 32), (2, 1, 16), (16, 4, 64), (4, 4, 80), (6, 1, 80), (12, 2, 96), (20, 1, 48), (32, 8, 128), (5, 5, 112), (8, 8, 256), (12, 1, 208), (40, 2, 128)]


@pytest.mark.parametrize("Hq, Hkv, h", HEADS)
@pytest.mark.parametrize("dt", [BF, HF])
def test_single_tokens_over_pages(Hq, Hkv, h, dt):
    for P in (8, 16, 64):
        attend_paged([1, 2, 8, 9, 31, 32, 33, 63, 64, 65, 127, 500], [1] * 12, Hq, Hkv, h, P, 0, 0, dt, seed=h + P)
        attend_paged([1, 40, 65, 300], [1] * 4, Hq, Hkv, h, P, 37, 3, dt, seed=h + P + 1)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (7, 0), (8, 8), (31, 2), (32, 33), (64, 5), (65, 64), (100, 130), (2, 300), (5000, 4)])
def test_single_tokens_with_windows_and_sinks(window, sinks):
    attend_paged([1, 2, 33, 64, 65, 66, 129, 257, 311, 1000, 1007], [1] * 11, 8, 2, 64, 16, window, sinks, BF, seed=window)


@pytest.mark.parametrize("S, Hq, Hkv, h, total", [(1, 8, 1, 128, 6000), (2, 4, 4, 64, 3001), (1, 2, 2, 256, 2500), (3, 32, 8, 128, 1111), (64, 32, 32, 80, 70), (200, 12, 12, 64, 90),
                                                  (300, 8, 8, 256, 40)])
def test_single_tokens_of_few_long_and_many_short_sequences(S, Hq, Hkv, h, total):
    """A job by one wave, by the waves of a block, and by several blocks whose parts are joined."""
    rng = random.Random(S)
    attend_paged([total] + [rng.randint(1, total) for _ in range(S - 1)], [1] * S, Hq, Hkv, h, 16, 0, 0, BF, seed=S)


def test_sequences_without_a_new_token_or_without_a_key():
    attend_paged([40, 7, 0, 33], [1, 0, 0, 1], 4, 2, 64, 8, 0, 0, BF, seed=3)
    # more new tokens than the cache holds: queries that see nothing have zeros and -infinity
    pages, table, kv = cache(random.Random(1), [3, 20], 8, 2, 64, BF, 5)
    q = rand(8, 9, 4, 64)
    out, lse = R.rlgen_window_attention_paged(q, pages, table, i32([0, 5, 9]), i32([3, 20]), 5, 20, 0, 0, 0.1)
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all()
    W.check("out", out[2:5], *W.attention(q[2:5], kv[0][0], kv[0][1], 0, 0, 0, 0.1, BF)["out"])
    W.check("out", out[5:], *W.attention(q[5:], kv[1][0], kv[1][1], 16, 0, 0, 0.1, BF)["out"])
    out, lse = R.rlgen_window_attention_paged(q[:1], pages, table[:1].contiguous(), i32([0, 1]), i32([0]), 1, 20, 0, 0, 0.1)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("Hq, Hkv, h", HEADS)
def test_chunks_over_pages(Hq, Hkv, h):
    attend_paged([5, 64, 130, 333, 70], [5, 2, 130, 40, 1], Hq, Hkv, h, 16, 0, 0, BF, seed=h)
    attend_paged([5, 64, 130, 333, 400], [5, 7, 30, 140, 3], Hq, Hkv, h, 8, 50, 5, HF, seed=h + 1)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (33, 2), (64, 70), (129, 4)])
def test_chunks_with_windows_and_sinks(window, sinks):
    attend_paged([300, 64, 1000, 129], [100, 64, 17, 2], 6, 3, 64, 32, window, sinks, BF, seed=window)


def test_a_cache_whose_offsets_pass_32_bits():
    """Pages more than 2^32 elements into the cache, for the write, the single token and the chunk."""
    Hq, Hkv, h, P = 8, 8, 128, 32
    n_pages = 2 ** 32 // (2 * Hkv * P * h) + 20
    pages = torch.empty((n_pages, 2, Hkv, P, h), dtype=BF, device="cuda")
    total, width = 100, 4
    table = i32([[n_pages - 1, 3, n_pages - 7, n_pages - 2]])
    rows = total
    qkv = rand(1, rows, 3 * Hq * h, dt=BF)
    one = torch.ones(h, device="cuda")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    slots = (table[0, (pos // P).long()].long() * P + pos.long() % P).int()
    q = R.rlgen_qk_norm_rope(qkv, one, one, 1e-5, None, pos, pages=pages, slots=slots)
    _, k, v = R.rlgen_qk_norm_rope(qkv, one, one, 1e-5, None, pos, n_kv_heads=Hkv)
    want = W.attention(q, k, v, 0, 0, 0, 0.09, BF)
    out, _ = R.rlgen_window_attention_paged(q, pages, table, i32([0, rows]), i32([total]), rows, total, 0, 0, 0.09)
    W.check("chunk", out, *want["out"])
    out, _ = R.rlgen_window_attention_paged(q[-1:], pages, table, i32([0, 1]), i32([total]), 1, total, 0, 0, 0.09)
    W.check("single token", out, *(x[-1:] for x in want["out"]))


def test_table_entries_outside_the_cache_are_not_followed():
    pages, table, kv = cache(random.Random(1), [40, 50], 8, 2, 64, BF, 5)
    table2 = table.clone()
    table2[0, 2], table2[0, 3] = 10 ** 9, -5
    q = rand(8, 2, 4, 64)
    for news, qq in (([1, 1], q), ([3, 3], rand(9, 6, 4, 64))):
        a = R.rlgen_window_attention_paged(qq, pages, table, starts_of(news), i32([40, 50]), news[0], 50, 0, 0, 0.1)
        b = R.rlgen_window_attention_paged(qq, pages, table2, starts_of(news), i32([40, 50]), news[0], 50, 0, 0, 0.1)
        assert torch.equal(a[0][news[0]:], b[0][news[0]:])


def test_a_captured_step_replays_as_it_runs():
    """Plan, norm with cache write and attention of a decode step in one graph: every replay against the eager step."""
    S, Hq, Hkv, h, P, steps = 5, 8, 2, 64, 16, 4
    ctx0, width = [3, 15, 16, 40, 0], 8
    rng = random.Random(9)
    table0, free = tables(rng, ctx0, [steps + 1] * S, P)
    table0 = [r + [-7] * (width - len(r)) for r in table0]
    n_pages = len(free) + sum(-(-c // P) for c in ctx0)
    pages0 = rand(2, n_pages, 2, Hkv, P, h)
    one, rope = torch.ones(h, device="cuda"), R.rlgen_rope_table(100, 32, 1e4)
    new, freed = i32([1] * S), i32(free)

    def step(st):
        plan = R.rlgen_plan_pages(st["lens"], new, P, freed, st["table"], S, st["head"])
        q = R.rlgen_qk_norm_rope(st["qkv"], one, one, 1e-5, rope, plan.positions, pages=st["pages"], slots=plan.slots)
        out, lse = R.rlgen_window_attention_paged(q, st["pages"], st["table"], plan.row_starts, plan.total_lens, 1, 100, 20, 2, 0.125)
        st["lens"].copy_(plan.total_lens)
        st["head"].copy_(plan.counts[1:2])
        return out, lse

    def fresh():
        return {"lens": i32(ctx0), "table": i32(table0), "head": i32([0]), "pages": pages0.clone(), "qkv": rand(50, S, (Hq + 2 * Hkv) * h)}

    eager, st = [], fresh()
    for i in range(steps):
        st["qkv"].copy_(rand(100 + i, S, (Hq + 2 * Hkv) * h))
        eager.append([x.clone() for x in step(st)])
    g_st = fresh()
    warm = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(g_st)
    for i in range(steps):
        g_st["qkv"].copy_(rand(100 + i, S, (Hq + 2 * Hkv) * h))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i][0]) and torch.equal(lse, eager[i][1]), i
    assert torch.equal(g_st["pages"], st["pages"]) and torch.equal(g_st["table"], st["table"])
