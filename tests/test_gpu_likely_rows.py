"""Rows whose likeliest token has more than half of the probability (S = sum exp((z - m) / T) between 1 and 2): the other terms keep their bits beside its 1.

T is the 32-bit number next to log2(e), so that the kernel's factor log2(e) / T is exactly 1, and logits are whole numbers: every term is a power of two, sums of the
others are exact in 32 bits (multiples of 2^-24 below 1).  What is left: the factor's own rounding, 0.23 U of exponents up to 24 log 2, 4 U of the others' sum; and the
logarithm with the three operations around it, 10 U.  The likeliest token stands first in its row and 31 terms of 2^-24 behind it in the same thread: added up beside
1 they would vanish one by one, 31 U of S or 16 to 470 U of its logarithm."""
import pytest
import torch

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
T = float(torch.tensor(1.4426950408889634, dtype=F32))


@pytest.mark.parametrize("dtype", [F32, BF, F16])
@pytest.mark.parametrize("rows, V, low", [(3, 50304, -19), (3, 50304, -18), (70, 50304, -17), (3, 50304, -16), (3, 8000, -16), (3, 8000, -14), (300, 2000, -14),
                                          (300, 2000, -12), (1, 70400, -18), (20, 70400, -17), (2, 262144, -20), (70, 131072, -18)])
@pytest.mark.parametrize("n", [0, 3])
def test_the_others_keep_their_bits(dtype, rows, V, low, n):
    z = torch.full((rows, V), float(low))
    # a thread's step of 32 values: pieces of 16 bytes, one to a thread in turn
    threads, piece = (64 if rows > 256 else 256), 4 if dtype is F32 else 8
    for u in range(32 // piece):
        z[:, u * threads * piece:u * threads * piece + piece] = -24
    z[:, 0] = 0
    others = torch.exp(z[0, 1:].double() / T)
    share = float(others.sum())
    assert 0.06 < share < 1
    log_sum = float(torch.log1p(torch.tensor(share, dtype=torch.float64)))
    H = log_sum - float((others * z[0, 1:].double() / T).sum()) / (1 + share)
    zd, tok = z.to(dtype).cuda(), torch.zeros(rows, dtype=torch.int32, device="cuda")
    got = R.rlgen_token_logprobs(zd, tok, T, n_top=n)
    for name, v, want, most in (("log sum", got.stats[:, 1], log_sum, 14), ("log-prob", got.logprobs, -log_sum, 14), ("entropy", got.entropy, H, 28)):
        off = (v.double() - want).abs() / abs(want)
        assert bool((off <= most * U).all()), (name, float(off.max()) / U)
    g = torch.ones(rows, device="cuda")
    d = R.rlgen_token_logprobs_backward(zd, tok, T, got.stats, g)
    # 1 - p: p = 1 / S, so its relative error is at most the log sum's, and that of the powers and factors around it
    want = share / (1 + share) / T
    half = 0 if dtype is F32 else torch.finfo(dtype).eps / 2
    assert bool(((d[:, 0].double() - want).abs() <= (half + 24 * U) * want).all())
