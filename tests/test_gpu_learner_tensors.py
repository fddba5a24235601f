"""Tensors that a kernel could not follow, in host memory, of another type or shape, or with gaps, are refused by the binding before anything is
launched."""
import pytest
import torch

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.gpu
rows, width, V = 60, 64, 70001
BF = torch.bfloat16


def calls():
    """Each operator with every tensor it takes by name."""
    x, gain, rng = torch.ones(rows, width, dtype=BF, device="cuda"), torch.ones(width, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    z, tok, f = torch.zeros(rows, V, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.ones(rows, device="cuda")
    out = R.rlgen_token_logprobs(z, tok, n_top=3)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    space = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    return {
        R.rlgen_add_rms_norm: dict(x=x, gain=gain, eps=1e-5, residual=x.clone(), drop_p=0.1, rng=rng,
                                   out=(x.clone(), x.to(torch.float8_e4m3fn), torch.empty(rows, 1, device="cuda"))),
        R.rlgen_add_rms_norm_backward: dict(h=x, gain=gain, eps=1e-5, dy=x.clone(), dh=x.clone(), drop_p=0.1, rng=rng, out=(x.clone(), x.clone(), gain.clone()),
                                            workspace=space(R.lib.rlgen_add_rms_norm_backward_workspace(rows, width))),
        R.rlgen_token_logprobs: dict(logits=z, tokens=tok, out=tuple(out), workspace=space(R.lib.rlgen_token_logprobs_workspace(0, rows, V, 3))),
        R.rlgen_token_logprobs_backward: dict(logits=z, tokens=tok, temperature=1.0, stats=out.stats, dlogprobs=f, entropy=out.entropy, dentropy=f.clone(),
                                              out=z.clone()),
        R.rlgen_dpo_pairs: dict(token_logprobs=f, ref_logprobs=f.clone(), row_starts=i32([0, 2, rows]), idx_pos=i32([0]), idx_neg=i32([1]), k=2, beta=0.1,
                                out=(torch.empty(1, device="cuda"), f.clone())),
    }


def variants(args):
    for name, value in args.items():
        if isinstance(value, torch.Tensor):
            yield name, value, lambda v: v
        elif isinstance(value, tuple):
            for i, v in enumerate(value):
                yield name, v, lambda v, i=i, value=value: tuple(v if j == i else x for j, x in enumerate(value))


def test_tensors_in_host_memory_are_refused():
    for f, args in calls().items():
        f(**args)
        torch.cuda.synchronize()
        for name, value, put in variants(args):
            with pytest.raises(AssertionError):
                f(**dict(args, **{name: put(value.cpu())}))


def test_other_types_and_shapes_are_refused():
    for f, args in calls().items():
        for name, value, put in variants(args):
            if name == "workspace":
                continue
            if value is not args.get("x") and value is not args.get("logits") and not (f is R.rlgen_add_rms_norm_backward and name in ("h", "dy")):
                with pytest.raises((AssertionError, KeyError)):
                    f(**dict(args, **{name: put(value.to(torch.float64))}))
            if value.dim() == 1 and name not in ("token_logprobs", "idx_pos"):
                with pytest.raises(AssertionError):
                    f(**dict(args, **{name: put(torch.cat([value, value]))}))
                with pytest.raises(AssertionError):
                    f(**dict(args, **{name: put(torch.stack([value, value], 1)[:, 0] if value.numel() > 1 else value[:0])}))
            if value.dim() == 2:
                with pytest.raises((AssertionError, R.RlgenError)):
                    f(**dict(args, **{name: put(torch.cat([value, value]))}))
                if value.shape[1] > 1:
                    with pytest.raises(AssertionError):
                        f(**dict(args, **{name: put(value.T.contiguous().T)}))


def test_workspaces_with_gaps_and_too_small_are_refused():
    for f, args in calls().items():
        if "workspace" in args:
            n = args["workspace"].numel()
            with pytest.raises(AssertionError):
                f(**dict(args, workspace=torch.empty(n, 2, dtype=torch.uint8, device="cuda")[:, 0]))
            with pytest.raises(R.RlgenError):
                f(**dict(args, workspace=args["workspace"][:n - 1]))
