"""fp16 gradients depend on their own sequence alone: what other sequences and rows that no sequence has hold, infinite or merely large,
changes no bit of them; and a row's dq keeps its precision beside larger or infinite rows of its own sequence."""
import math

import pytest
import torch

import window_reference as W
from test_gpu_operators import HF, R, i32, rand

pytestmark = pytest.mark.gpu
SMALL = 2.0 ** -18


def gradients(x, st, longest, window, sinks, scale):
    q, k, v, do = x
    out, lse = R.rlgen_window_attention(q, k, v, st, longest, window, sinks, scale)
    return out, lse, R.rlgen_window_attention_backward(q, k, v, out, lse, do, st, longest, window, sinks, scale)


def inputs(rows, Hq, Hkv, h, size, seed):
    q, k, v = (rand(seed + i, rows, n, h, dt=HF) for i, n in enumerate((Hq, Hkv, Hkv)))
    return [q, k, v, (rand(seed + 9, rows, Hq, h, dt=torch.float32) * size).half()]


@pytest.mark.parametrize("Hq, Hkv, h, window, sinks", [(2, 1, 64, 0, 0), (4, 4, 80, 70, 3), (4, 2, 128, 0, 0), (2, 2, 256, 40, 2), (8, 1, 32, 20, 0)])
@pytest.mark.parametrize("beside", ["infinite dout", "infinite v", "large dout", "large v and dout", "NaN"])
def test_another_sequence_changes_no_bit(Hq, Hkv, h, window, sinks, beside):
    lens, rows = [150, 60, 97], 320                      # (13 rows belong to no sequence)
    x = inputs(rows, Hq, Hkv, h, SMALL, h)
    st, scale = i32([0, 150, 210, 307]), 1 / math.sqrt(h)
    clean = gradients(x, st, 150, window, sinks, scale)
    at = 0
    for n in lens:
        part = slice(at, at + n)
        want = W.attention(x[0][part], x[1][part], x[2][part], 0, window, sinks, scale, HF, x[3][part])
        for name, g in zip(("dq", "dk", "dv"), clean[2]):
            W.check(name, g[part], *want[name])
        at += n
    value = {"infinite dout": (None, math.inf), "infinite v": (math.inf, None), "large dout": (None, 3e4), "large v and dout": (1000.0, 1.0),
             "NaN": (math.nan, math.nan)}[beside]
    for where in (slice(150, 210), slice(307, 320)):      # another sequence, rows of none
        y = [t.clone() for t in x]
        for t, f in zip(y[2:], value):
            if f is not None:
                t[where, :, 5] = f
        out, lse, got = gradients(y, st, 150, window, sinks, scale)
        keep = torch.ones(rows, dtype=torch.bool, device="cuda")
        keep[150:210] = keep[307:] = False
        for name, a, b in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *got), (*clean[:2], *clean[2])):
            assert torch.equal(a[keep], b[keep]), (name, where)


@pytest.mark.parametrize("window, sinks", [(0, 0), (50, 2)])
def test_rows_beyond_the_callers_bound_change_no_bit(window, sinks):
    Hq, Hkv, h, bound, scale = 4, 2, 64, 100, 0.125
    x = inputs(360, Hq, Hkv, h, SMALL, 3)
    st = i32([0, 100, 300, 360])
    a = gradients(x, st, bound, window, sinks, scale)
    y = [t.clone() for t in x]
    y[2][200:300], y[3][200:300] = math.inf, 6e4
    b = gradients(y, st, bound, window, sinks, scale)
    keep = torch.ones(360, dtype=torch.bool, device="cuda")
    keep[200:300] = False
    for name, u, w in zip(("dq", "dk", "dv"), a[2], b[2]):
        assert torch.equal(u[keep], w[keep]), name


@pytest.mark.parametrize("Hq, Hkv, h, window, sinks", [(2, 1, 64, 0, 0), (4, 4, 80, 70, 3), (4, 2, 128, 0, 0), (2, 2, 256, 40, 2)])
@pytest.mark.parametrize("value", [math.inf, 6e4])
def test_a_row_keeps_its_precision_beside_larger_ones(Hq, Hkv, h, window, sinks, value):
    """dq of a row is the product of its own dout, so one outlier in another row's dout leaves it as exact as it was."""
    n, row, scale = 200, 187, 1 / math.sqrt(h)
    x = inputs(n, Hq, Hkv, h, SMALL, 40 + h)
    want = W.attention(*x[:3], 0, window, sinks, scale, HF, x[3])["dq"]
    x[3][row, :, 7] = value
    dq = gradients(x, i32([0, n]), n, window, sinks, scale)[2][0]
    keep = [i for i in range(n) if i != row]
    W.check("dq", dq[keep], want[0][keep], want[1][keep])


@pytest.mark.parametrize("Hq, Hkv, h, window, sinks", [(2, 1, 64, 0, 0), (4, 4, 80, 250, 3), (4, 2, 128, 0, 0), (2, 2, 256, 200, 130), (8, 1, 32, 0, 0)])
@pytest.mark.parametrize("first", [True, False])
def test_small_values_beside_large_ones(Hq, Hkv, h, window, sinks, first):
    """What is subtracted in dS comes from all keys in sight: where they are of very different sizes, dS of the small ones stays in the type's range."""
    n, scale = 420, 1 / math.sqrt(h)
    x = inputs(n, Hq, Hkv, h, 1.0, 60 + h)
    size = torch.where((torch.arange(n) < 150) == first, 2.0 ** -10, 2.0 ** 8)[:, None, None].cuda()
    x[2] = (x[2].float() * size).half()
    want = W.attention(*x[:3], 0, window, sinks, scale, HF, x[3])
    out, lse, got = gradients(x, i32([0, n]), n, window, sinks, scale)
    for name, g in zip(("dq", "dk", "dv"), got):
        W.check(name, g, *want[name])
