"""Gradients of keys whose queries are parted over blocks (few kv heads, long sequences), against the plain 64-bit form
(window_reference) with the bounds that it derives from the types."""
import pytest
import torch

from test_gpu_operators import BF, HF, R, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens, Hq, Hkv, h, window, sinks", [
    ([700, 513], 8, 1, 64, 0, 0), ([1200], 12, 1, 96, 0, 0), ([0, 900, 1, 130], 5, 1, 80, 0, 0), ([1100], 4, 2, 128, 0, 0), ([1400], 8, 1, 32, 300, 0),
    ([1400, 40], 8, 1, 64, 600, 5), ([1300], 8, 1, 48, 900, 200), ([1500], 4, 1, 256, 0, 0), ([1300], 16, 2, 112, 40, 4), ([640], 40, 1, 16, 640, 0)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_gradients_of_few_long_sequences(lens, Hq, Hkv, h, window, sinks, dt):
    attend(lens, Hq, Hkv, h, window, sinks, dt, seed=sum(lens) + h)


def test_parted_gradients_are_the_same_every_time():
    q, k, v, st, out, lse, do, got = attend([900, 650], 8, 1, 64, 500, 3, BF)
    for _ in range(3):
        again = R.rlgen_window_attention_backward(q, k, v, out, lse, do, st, 900, 500, 3, 0.125)
        assert all(torch.equal(got[name], x) for name, x in zip(("dq", "dk", "dv"), again))


@pytest.mark.parametrize("h, window, sinks", [(64, 0, 0), (128, 200, 3), (256, 0, 0)])
def test_rows_beyond_the_callers_bound_are_left_alone(h, window, sinks):
    """A sequence longer than max_len: its first max_len rows are computed as if it ended there, the others and their gradients not."""
    bound, lens, Hq, Hkv = 600, [300, 1500, 40], 4, 1
    q, k, v, st, out, lse, do, got = attend(lens, Hq, Hkv, h, window, sinks, BF)
    cut = torch.cat([torch.arange(n)[:bound] + at for at, n in zip([0, 300, 1800], lens)]).cuda()
    qc, kc, vc, doc = (x[cut].contiguous() for x in (q, k, v, do))
    stc = torch.tensor([0, 300, 900, 940], dtype=torch.int32, device="cuda")
    out_c, lse_c = R.rlgen_window_attention(qc, kc, vc, stc, bound, window, sinks, 0.1)
    grads_c = R.rlgen_window_attention_backward(qc, kc, vc, out_c, lse_c, doc, stc, bound, window, sinks, 0.1)
    into = [torch.full((sum(lens), H, h), 7.0, dtype=BF, device="cuda") for H in (Hq, Hq, Hkv, Hkv)]
    lse_b = torch.full((sum(lens), Hq), 7.0, device="cuda")
    R.rlgen_window_attention(q, k, v, st, bound, window, sinks, 0.1, out=(into[0], lse_b))
    R.rlgen_window_attention_backward(q, k, v, into[0], lse_b, do, st, bound, window, sinks, 0.1, grads=into[1:])
    beyond = torch.ones(sum(lens), dtype=torch.bool, device="cuda")
    beyond[cut] = False
    assert all(bool((x[beyond] == 7.0).all()) for x in [*into, lse_b])
    assert all(torch.equal(x[cut], want) for x, want in zip([*into[:2], lse_b], [out_c, grads_c[0], lse_c]))
    # (the parts of a tile of keys depend on all rows, so two sums may differ by fp32's roundings and then by one of bf16)
    for x, want in zip(into[2:], grads_c[1:]):
        d, w = (x[cut].double() - want.double()).abs(), want.double().abs()
        assert bool((d <= 2.0 ** -7 * w + 2.0 ** -12 * w.max()).all())
