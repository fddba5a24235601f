"""Sizes past 32 bits, which the C entry points could not tell from smaller ones, are refused by the binding before anything else.  Tensors without
memory stand for ones too large to make here; where there is a device they are refused for not being on it."""
import pytest
import torch

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-only checks")
MANY = 2 ** 32 + 5


def meta(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("shape", [(MANY, 8), (2 ** 31, 8), (1, MANY)])
def test_rows_and_widths(shape):
    x, gain = meta(*shape), meta(shape[1], dtype=torch.float32)
    rows, one = shape[0], meta(shape[0], dtype=torch.float32)
    with pytest.raises(AssertionError):
        R.rlgen_add_rms_norm(x, gain, 1e-5, out=(x, x))
    with pytest.raises(AssertionError):
        R.rlgen_add_rms_norm_backward(x, gain, 1e-5, x, out=(x, x, gain), workspace=x)
    with pytest.raises(AssertionError):
        R.rlgen_token_logprobs(x, out=(None, None, meta(rows, 2, dtype=torch.float32), None, None), workspace=x)
    with pytest.raises(AssertionError):
        R.rlgen_token_logprobs_backward(x, one.to(torch.int32), 1.0, meta(rows, 2, dtype=torch.float32), one, out=x)


@pytest.mark.parametrize("rows, B, k", [(MANY, 2, 2), (9, MANY, 1), (9, 1, MANY)])
def test_pairs(rows, B, k):
    lp, starts, idx = meta(rows, dtype=torch.float32), meta(B * k + 1, dtype=torch.int32), meta(B, dtype=torch.int32)
    with pytest.raises(AssertionError):
        R.rlgen_dpo_pairs(lp, lp, starts, idx, idx, k, 0.1, out=(meta(B, dtype=torch.float32), lp))


@pytest.mark.parametrize("scale_group", [2 ** 32, 2 ** 32 + 64, -2 ** 32])
def test_scale_groups(scale_group):
    x, gain = meta(3, 64), meta(64, dtype=torch.float32)
    with pytest.raises(AssertionError):
        R.rlgen_add_rms_norm(x, gain, 1e-5, scale_group=scale_group, out=(x, x.to(torch.float8_e4m3fn), meta(3, 1, dtype=torch.float32)))
