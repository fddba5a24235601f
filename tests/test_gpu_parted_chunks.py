"""A few new rows behind long contexts, whose keys are parted over blocks and joined, against the plain 64-bit form (window_reference) with
the bounds that it derives from the types."""
import math
import random

import pytest
import torch

import window_reference as W
from test_gpu_operators import BF, HEADS, HF, R, attend_paged, cache, i32, rand, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq, Hkv, h", HEADS)
@pytest.mark.parametrize("dt", [BF, HF])
def test_few_rows_of_every_head_size(Hq, Hkv, h, dt):
    attend_paged([1501], [3], Hq, Hkv, h, 16, 0, 0, dt, seed=h)
    attend_paged([900, 5, 0, 2000, 1], [2, 5, 0, 9, 1], Hq, Hkv, h, 8, 0, 0, dt, seed=h + 1)


@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 2), (40, 0), (700, 5), (600, 300), (1999, 1), (5000, 4)])
@pytest.mark.parametrize("news", [[2, 7, 1], [65, 3, 30]])
def test_few_rows_with_windows_and_sinks(window, sinks, news):
    attend_paged([2000, 1100, 31], news, 8, 2, 64, 32, window, sinks, BF, seed=window)


def test_a_call_without_the_workspace_and_with_it():
    totals, news = [3000, 1234], [4, 2]
    pages, table, kv = cache(random.Random(3), totals, 16, 2, 64, BF, 3)
    q = rand(9, sum(news), 8, 64)
    size = R.lib.rlgen_window_attention_chunk_workspace(8, 2, 64, 2, 4, 3000, 0, 0)
    assert size > 0
    args = (q, pages, table, starts_of(news), i32(totals), 4, 3000, 0, 0, 0.125)
    parted = R.rlgen_window_attention_paged(*args)
    held = R.rlgen_window_attention_paged(*args, workspace=torch.full((size,), 255, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(parted, held))              # (nothing is read that the call did not write)
    whole = R.rlgen_window_attention_paged(*args, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    at = 0
    for i, n in enumerate(news):
        want = W.attention(q[at:at + n], kv[i][0], kv[i][1], totals[i] - n, 0, 0, 0.125, BF)
        for got in (parted, whole):
            W.check("out", got[0][at:at + n], *want["out"])
            W.check("lse", got[1][at:at + n], *want["lse"])
        at += n


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_only_the_last_row_sees_reaches_no_other(bad):
    total, n = 1500, 4
    pages, table, kv = cache(random.Random(5), [total], 16, 2, 64, BF, 5)
    q = rand(6, n, 4, 64)
    args = (q, pages, table, starts_of([n]), i32([total]), n, total, 0, 0, 0.125)
    clean = R.rlgen_window_attention_paged(*args)
    page, at = int(table[0, (total - 1) // 16]), (total - 1) % 16
    pages[page, 1, 1, at, 7] = bad                                           # one dim of the last token's value, second kv head
    out, lse = R.rlgen_window_attention_paged(*args)
    want = W.attention(q, kv[0][0], kv[0][1], total - n, 0, 0, 0.125, BF)
    W.check("rows before it", out[:-1], *(x[:-1] for x in want["out"]))
    W.check("lse", lse, *want["lse"])
    assert torch.equal(out[-1, :2], clean[0][-1, :2])
    assert bool((out[-1, 2:, 7].isnan() if bad != bad else out[-1, 2:, 7] == bad).all())
    keep = [d for d in range(64) if d != 7]
    W.check("the last row's other dims", out[-1:, :, keep], *(x[-1:, :, keep] for x in want["out"]))
