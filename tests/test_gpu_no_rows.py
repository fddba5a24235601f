"""Passes without any row, as a rank or a step without work makes them: every operator returns, and sums over no row are zero."""
import pytest
import torch

from test_gpu_operators import BF, HF, R, i32, rand

pytestmark = pytest.mark.gpu
Hq, Hkv, h = 4, 2, 64


@pytest.mark.parametrize("dt", [BF, HF])
def test_norm_rope_without_rows(dt):
    one, pos = torch.ones(h, device="cuda"), i32([])
    qkv = torch.empty(0, (Hq + 2 * Hkv) * h, dtype=dt, device="cuda")
    q, k, v = R.rlgen_qk_norm_rope(qkv, one, one, 1e-5, None, pos, n_kv_heads=Hkv)
    assert q.shape == (0, Hq, h) and k.shape == v.shape == (0, Hkv, h)
    pages = rand(1, 3, 2, Hkv, 8, h, dt=dt)
    before = pages.clone()
    q = R.rlgen_qk_norm_rope(qkv, one, one, 1e-5, R.rlgen_rope_table(9, 32, 1e4), pos, pages=pages, slots=i32([]))
    assert q.shape == (0, Hq, h) and torch.equal(pages, before)
    grads = [torch.full((h,), 7.0, device="cuda") for _ in range(2)]
    dqkv, dqg, dkg = R.rlgen_qk_norm_rope_backward(qkv, one, one, 1e-5, None, pos, q, k, v, out=(torch.empty_like(qkv), *grads))
    assert dqkv.shape == qkv.shape and bool((dqg == 0).all()) and bool((dkg == 0).all())


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("S", [1, 3])
def test_attention_without_rows(dt, S):
    q, k, v = (torch.empty(0, n, h, dtype=dt, device="cuda") for n in (Hq, Hkv, Hkv))
    st = i32([0] * (S + 1))
    out, lse = R.rlgen_window_attention(q, k, v, st, 1, 20, 2, 0.1)
    assert out.shape == (0, Hq, h) and lse.shape == (0, Hq)
    grads = R.rlgen_window_attention_backward(q, k, v, out, lse, out, st, 1, 20, 2, 0.1)
    assert [g.shape for g in grads] == [q.shape, k.shape, v.shape]


@pytest.mark.parametrize("S", [1, 3])
@pytest.mark.parametrize("max_new", [1, 5])
def test_a_step_in_which_no_request_adds_a_token(S, max_new):
    free, table = i32(list(range(8))), torch.full((S, 2), -1, dtype=torch.int32, device="cuda")
    plan = R.rlgen_plan_pages(i32([0] * S), i32([0] * S), 8, free, table, 0)
    pages = rand(1, 8, 2, Hkv, 8, h)
    out, lse = R.rlgen_window_attention_paged(torch.empty(0, Hq, h, dtype=BF, device="cuda"), pages, table, plan.row_starts, plan.total_lens, max_new, 16,
                                              0, 0, 0.1)
    assert out.shape == (0, Hq, h) and lse.shape == (0, Hq)
