"""Pages that a request lacks (an entry outside the cache, as the plan leaves it when the free list has run out): their tokens are seen by
nobody, and no other page's tokens stand in for them."""
import math
import random

import pytest
import torch

import window_reference as W
from test_gpu_operators import BF, HF, R, cache, i32, rand, starts_of

pytestmark = pytest.mark.gpu
real_seen = W.seen


def run(monkeypatch, totals, news, holes, Hq, Hkv, h, P, window, sinks, dt, seed, bad=(-1, 10 ** 9), workspace=None):
    """holes: for each sequence the places in its table that are outside the cache."""
    pages, table, kv = cache(random.Random(seed), totals, P, Hkv, h, dt, seed)
    pages = torch.where(pages.isnan(), torch.full_like(pages, 50.0), pages)      # (what stands in page 0 would show)
    for s, at in enumerate(holes):
        for i, e in enumerate(at):
            table[s, e] = bad[i % len(bad)]
    q, scale = rand(seed + 99, sum(news), Hq, h, dt=dt), 1 / math.sqrt(h)
    out, lse = R.rlgen_window_attention_paged(q, pages, table, starts_of(news), i32(totals), max(news), max(totals), window, sinks, scale,
                                              workspace=workspace)
    at = 0
    for s, (t, n) in enumerate(zip(totals, news)):
        there = torch.ones(max(t, 1), dtype=torch.bool)
        for e in holes[s]:
            there[e * P:(e + 1) * P] = False
        monkeypatch.setattr(W, "seen", lambda pos, T, w, k: real_seen(pos, T, w, k) & there[None, :T])
        want = W.attention(q[at:at + n], kv[s][0], kv[s][1], t - n, window, sinks, scale, dt)
        W.check(f"out of sequence {s}", out[at:at + n], *want["out"])
        W.check(f"lse of sequence {s}", lse[at:at + n], *want["lse"])
        at += n
    return out, lse


SHAPES = [(4, 4, 32), (8, 2, 64), (6, 1, 80), (12, 2, 96), (8, 2, 128), (2, 2, 256)]


@pytest.mark.parametrize("Hq, Hkv, h", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
def test_single_tokens(monkeypatch, Hq, Hkv, h, dt):
    for P in (8, 32):
        run(monkeypatch, [300, 65, 40, 9], [1] * 4, [[0, 3], [1], [], [0]], Hq, Hkv, h, P, 0, 0, dt, h + P)
    run(monkeypatch, [300, 65, 129], [1] * 3, [[0, 18], [3], [7, 8]], Hq, Hkv, h, 16, 37, 3, dt, h + 1)


def test_single_tokens_of_many_sequences(monkeypatch):
    """A job to a wave."""
    run(monkeypatch, [40 + i % 30 for i in range(70)], [1] * 70, [[i % 3] if i % 2 else [] for i in range(70)], 32, 32, 64, 16, 0, 0, BF, 5)


def test_a_sequence_without_any_page(monkeypatch):
    for news in ([1, 1], [3, 5]):
        out, lse = run(monkeypatch, [30, 50], news, [[0, 1], []], 4, 2, 64, 16, 0, 0, BF, 7)
        assert bool((out[:news[0]] == 0).all()) and bool((lse[:news[0]] == -math.inf).all())


@pytest.mark.parametrize("Hq, Hkv, h", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
def test_chunks(monkeypatch, Hq, Hkv, h, dt):
    none = torch.empty(16, dtype=torch.uint8, device="cuda")
    run(monkeypatch, [330, 64, 150], [40, 7, 150], [[0, 2, 5], [], [3]], Hq, Hkv, h, 16, 0, 0, dt, h, workspace=none)
    run(monkeypatch, [330, 64, 400], [140, 2, 30], [[0, 40], [7], [45, 44]], Hq, Hkv, h, 8, 50, 5, dt, h + 1, workspace=none)


@pytest.mark.parametrize("window, sinks", [(0, 0), (700, 5)])
def test_parted_chunks(monkeypatch, window, sinks):
    assert R.lib.rlgen_window_attention_chunk_workspace(8, 2, 64, 2, 9, 2000, window, sinks) > 0
    run(monkeypatch, [2000, 900], [9, 2], [[0, 60, 61, 120], [20]], 8, 2, 64, 16, window, sinks, BF, 11)


def test_a_row_that_is_computed_key_by_key(monkeypatch):
    """A NaN that one row alone sees has its tile computed again; missing pages stay unseen there too."""
    totals, news, P = [100], [4], 16
    pages, table, kv = cache(random.Random(2), totals, P, 1, 64, BF, 2)
    pages = torch.where(pages.isnan(), torch.full_like(pages, 50.0), pages)
    page = int(table[0, 99 // P])
    table[0, 1] = -1
    q = rand(4, 4, 2, 64)
    pages[page, 1, 0, 99 % P, 7] = math.nan
    for ws in (None, torch.empty(16, dtype=torch.uint8, device="cuda")):
        out, _ = R.rlgen_window_attention_paged(q, pages, table, i32([0, 4]), i32(totals), 4, 100, 0, 0, 0.125, workspace=ws)
        there = torch.ones(100, dtype=torch.bool)
        there[P:2 * P] = False
        monkeypatch.setattr(W, "seen", lambda pos, T, w, k: real_seen(pos, T, w, k) & there[None, :T])
        want = W.attention(q, kv[0][0], kv[0][1], 96, 0, 0, 0.125, BF)["out"]
        W.check("rows before it", out[:3], *(x[:3] for x in want))
        keep = [d for d in range(64) if d != 7]
        W.check("its other dims", out[3:, :, keep], *(x[3:, :, keep] for x in want))
        assert bool(out[3, :, 7].isnan().all())
