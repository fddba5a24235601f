"""Tensors that a kernel could not follow, in host memory or with gaps, are refused by the binding before anything is launched."""
import pytest
import torch

from test_gpu_operators import BF, R, i32, rand

pytestmark = pytest.mark.gpu
Hq, Hkv, h, rows, S = 4, 2, 64, 6, 2


def calls():
    """Each operator with every tensor it takes by name."""
    st, total = i32([0, 2, rows]), i32([2, 4])
    one, pos = torch.ones(h, device="cuda"), i32(list(range(rows)))
    rope, table = R.rlgen_rope_table(9, 32, 1e4), i32([[0], [1]])
    qkv, pages = rand(1, rows, (Hq + 2 * Hkv) * h), rand(2, 3, 2, Hkv, 8, h)
    q, k, v, do = (rand(3 + i, rows, n, h) for i, n in enumerate((Hq, Hkv, Hkv, Hq)))
    lse = torch.empty(rows, Hq, device="cuda")

    def space(n):
        return torch.empty(n, dtype=torch.uint8, device="cuda")

    norm = dict(qkv=qkv, q_gain=one, k_gain=one.clone(), eps=1e-5, rope=rope, positions=pos)
    rest = dict(row_starts=st, max_len=4, window=0, sinks=0, scale=0.1)
    back = space(R.lib.rlgen_window_attention_backward_workspace(rows, Hq, Hkv, h, S, 4, 0, 0))
    return {
        R.rlgen_plan_pages: dict(ctx_lens=i32([0, 0]), new_lens=total, page_size=8, free_pages=i32([0, 1]), page_table=table, max_rows=rows, free_head=i32([0]),
                                 out=(total.clone(), st.clone(), pos.clone(), pos.clone(), i32([0] * 4))),
        R.rlgen_qk_norm_rope: dict(norm, pages=pages, slots=pos, out=q),
        R.rlgen_qk_norm_rope_backward: dict(norm, dq=q, dk=k, dv=v, out=(qkv.clone(), one.clone(), one.clone()),
                                            workspace=space(R.lib.rlgen_qk_norm_rope_backward_workspace(rows, h))),
        R.rlgen_window_attention: dict(rest, q=q, k=k, v=v, out=(do.clone(), lse)),
        R.rlgen_window_attention_backward: dict(rest, q=q, k=k, v=v, out=do.clone(), lse=lse, dout=do, grads=(q.clone(), k.clone(), v.clone()), workspace=back),
        R.rlgen_window_attention_paged: dict(q=q, pages=pages, page_table=table, row_starts=st, total_lens=total, max_new=4, max_total=4, window=0, sinks=0,
                                             scale=0.1, out=(do.clone(), lse), workspace=space(16)),
    }


def test_tensors_in_host_memory_are_refused():
    for f, args in calls().items():
        f(**args)
        torch.cuda.synchronize()
        for name, value in args.items():
            if isinstance(value, torch.Tensor):
                with pytest.raises(AssertionError):
                    f(**dict(args, **{name: value.cpu()}))
            elif isinstance(value, tuple):
                for i in range(len(value)):
                    with pytest.raises(AssertionError):
                        f(**dict(args, **{name: tuple(x.cpu() if j == i else x for j, x in enumerate(value))}))
    with pytest.raises(AssertionError):
        R.rlgen_rope_table(9, 32, 1e4, device="cpu")


def test_workspaces_with_gaps_are_refused():
    for f, args in calls().items():
        if "workspace" in args:
            n = max(args["workspace"].numel(), 64)
            with pytest.raises(AssertionError):
                f(**dict(args, workspace=torch.empty(n, 2, dtype=torch.uint8, device="cuda")[:, 0]))


def test_statistics_of_another_type_or_shape_are_refused():
    a = calls()
    bad = [(R.rlgen_qk_norm_rope, "q_gain", torch.ones(h, device="cuda", dtype=BF)), (R.rlgen_qk_norm_rope, "k_gain", torch.ones(h + 16, device="cuda")),
           (R.rlgen_qk_norm_rope, "rope", torch.ones(9, 16, 2, device="cuda", dtype=torch.float64)),
           (R.rlgen_qk_norm_rope, "rope", torch.ones(9, 2, 16, device="cuda").transpose(1, 2)),
           (R.rlgen_window_attention_backward, "lse", torch.ones(rows, Hq + 1, device="cuda")),
           (R.rlgen_window_attention_backward, "lse", torch.ones(Hq, rows, device="cuda").T)]
    for f, name, value in bad:
        with pytest.raises(AssertionError):
            f(**dict(a[f], **{name: value}))
