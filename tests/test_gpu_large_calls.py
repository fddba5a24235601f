"""Calls near the sizes that one launch holds: a decode step of thousands of sequences, one packed sequence of hundreds of thousands of rows."""
import pytest
import torch

import window_reference as W
from test_gpu_operators import BF, R, i32, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S, Hq, Hkv", [(4096, 32, 32), (16384, 8, 8)])
def test_a_decode_step_of_thousands_of_sequences(S, Hq, Hkv):
    """Each sequence has the result that it has in a call of 512."""
    h, P = 16, 8
    g = torch.Generator(device="cuda").manual_seed(S)
    pages = torch.randn(S, 2, Hkv, P, h, generator=g, device="cuda").to(BF)
    table = torch.randperm(S, generator=g, device="cuda").int().view(S, 1)
    total = torch.randint(1, P + 1, (S,), generator=g, device="cuda").int()
    q = torch.randn(S, Hq, h, generator=g, device="cuda").to(BF)
    starts = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    out, lse = R.rlgen_window_attention_paged(q, pages, table, starts, total, 1, P, 0, 0, 0.25)
    for i in range(0, S, 512):
        part = slice(i, i + 512)
        o, l = R.rlgen_window_attention_paged(q[part], pages, table[part], starts[:513], total[part], 1, P, 0, 0, 0.25)
        assert torch.equal(o, out[part]) and torch.equal(l, lse[part])
    for s in (0, 1, S // 2, S - 1):
        n = int(total[s])
        k, v = (pages[int(table[s, 0]), i, :, :n].transpose(0, 1) for i in (0, 1))
        want = W.attention(q[s:s + 1], k, v, n - 1, 0, 0, 0.25, BF)
        W.check("out", out[s:s + 1], *want["out"])
        W.check("lse", lse[s:s + 1], *want["lse"])


def test_one_sequence_of_a_quarter_of_a_million_rows():
    """With a window a run of rows depends on the rows just before it, and a run of keys on those just behind it."""
    rows, Hq, Hkv, h, window, scale = 262144, 64, 8, 16, 50, 0.25
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (torch.empty(rows, n, h, dtype=BF, device="cuda").normal_(generator=g) for n in (Hq, Hkv, Hkv, Hq))
    st = i32([0, rows])
    out, lse = R.rlgen_window_attention(q, k, v, st, rows, window, 0, scale)
    dq, dk, dv = R.rlgen_window_attention_backward(q, k, v, out, lse, do, st, rows, window, 0, scale)
    for at in (0, 100000, rows - 200):
        part = slice(at, at + 200)
        want = W.attention(q[part], k[part], v[part], 0, window, 0, scale, BF, do[part])
        first, last = (0 if at == 0 else window - 1), (200 if at == rows - 200 else 200 - window)
        for name, got in (("out", out), ("lse", lse), ("dq", dq)):
            W.check(name, got[part][first:], *(x[first:] for x in want[name]))
        for name, got in (("dk", dk), ("dv", dv)):
            W.check(name, got[part][first:last], *(x[first:last] for x in want[name]))
