"""The pairs' loss where log-probs are not finite or the step overflows (a masked token's log-prob is -infinity): only the pair's own loss and
rows may show it.  Bounds as for finite values: outputs are rounded once to 32 bits, the step once more before its sign."""
import pytest
import torch

import learner_reference as L

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF, NAN, LN2 = float("inf"), float("nan"), 0.6931471805599453
STARTS = [0, 4, 9, 11, 14, 20, 27]                               # two prompts of three sequences
SEQ = [slice(a, b) for a, b in zip(STARTS, STARTS[1:])]


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def logprobs():
    g = torch.Generator().manual_seed(1)
    ref = -torch.rand(27, generator=g) * 4
    return ref + 0.2 * torch.randn(27, generator=g), ref


def call(pol, ref, pos, neg, beta=0.1, weight=1.0):
    loss, grad = torch.empty(2, device="cuda"), torch.full((27,), 3.0, device="cuda")
    R.rlgen_dpo_pairs(pol.cuda(), ref.cuda(), i32(STARTS), i32(pos), i32(neg), 3, beta, weight, out=(loss, grad))
    return loss.cpu(), grad.cpu()


def second_prompt_is_right(loss, grad, pos, neg, beta=0.1, weight=1.0):
    """The prompt without unusual values."""
    pol, ref = logprobs()
    want, dwant = L.dpo_pairs(pol, ref, STARTS, pos, neg, 3, beta, weight)
    assert abs(float(loss[1]) - float(want[1])) <= 2 * U * float(want[1])
    assert bool(((grad[11:].double() - dwant[11:]).abs() <= 2 * U * dwant[11:].abs()).all())


@pytest.mark.parametrize("pol_value, ref_value", [(-INF, -INF), (NAN, -1.0), (-1.0, NAN), (INF, INF)])
@pytest.mark.parametrize("where", ["chosen", "rejected"])
def test_an_undefined_sum_stays_in_its_pair(pol_value, ref_value, where):
    pol, ref = logprobs()
    row = 5 if where == "chosen" else 10
    pol[row], ref[row] = pol_value, ref_value
    loss, grad = call(pol, ref, [1, 0], [2, 1])
    assert torch.isnan(loss[0]) and torch.isnan(grad[SEQ[1]]).all() and torch.isnan(grad[SEQ[2]]).all()
    assert (grad[SEQ[0]] == 0).all()                             # the prompt's other sequence
    second_prompt_is_right(loss, grad, [1, 0], [2, 1])


@pytest.mark.parametrize("row, loss_is, share", [(5, INF, 1.0), (10, 0.0, 0.0)])
def test_an_infinite_difference_has_the_limits_of_loss_and_gradient(row, loss_is, share):
    """The policy gives a token of y+ (row 5) or y- (row 10) no chance: sigmoid(-beta x) is 1 or 0."""
    pol, ref = logprobs()
    pol[row] = -INF
    loss, grad = call(pol, ref, [1, 0], [2, 1], beta=0.25, weight=0.5)
    assert float(loss[0]) == loss_is and (grad[SEQ[0]] == 0).all()
    assert (grad[SEQ[1]] == -0.125 * share).all() and (grad[SEQ[2]] == 0.125 * share).all()
    second_prompt_is_right(loss, grad, [1, 0], [2, 1], 0.25, 0.5)


@pytest.mark.parametrize("value", [-INF, INF, NAN])
@pytest.mark.parametrize("pos, neg", [(1, 1), (2 ** 31 - 1, 2)])
def test_the_same_index_twice_is_no_difference_whatever_its_log_probs(value, pos, neg):
    """(An index beyond the sequences is the last one.)"""
    pol, ref = logprobs()
    pol[SEQ[1]], pol[SEQ[2]] = value, value
    loss, grad = call(pol, ref, [pos, 0], [neg, 1])
    assert abs(float(loss[0]) - LN2) <= U and (grad[:11] == 0).all()
    second_prompt_is_right(loss, grad, [pos, 0], [neg, 1])


def test_a_step_that_overflows_stays_in_its_pair():
    """weight beta beyond 32 bits: infinite on the pair's rows, 0 on the others'."""
    pol, ref = logprobs()
    loss, grad = call(pol, ref, [1, 0], [2, 0], beta=1e-10, weight=3e38)
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all()
    zero = torch.zeros(27)
    loss, grad = call(zero, zero, [1, 0], [2, 0], beta=1e30, weight=1e30)
    assert (grad[SEQ[1]] == -INF).all() and (grad[SEQ[2]] == INF).all()
    assert (grad[SEQ[0]] == 0).all() and (grad[11:] == 0).all() and bool(((loss - LN2).abs() <= U).all())


def test_a_masked_token_from_logits_to_gradients():
    """As the learner runs it: the chosen sequence has a token that both models mask; the third sequence and the other prompt keep their gradients."""
    g = torch.Generator().manual_seed(2)
    z, zr = torch.randn(27, 50, generator=g), torch.randn(27, 50, generator=g)
    tokens = torch.randint(0, 50, (27,), generator=g)
    z[6, tokens[6]] = zr[6, tokens[6]] = -INF
    tok = tokens.int().cuda()
    lp, ref = R.rlgen_token_logprobs(z.cuda(), tok, entropy=False), R.rlgen_token_logprobs(zr.cuda(), tok, entropy=False)
    assert float(lp.logprobs[6]) == -INF
    _, dlp = R.rlgen_dpo_pairs(lp.logprobs, ref.logprobs, i32(STARTS), i32([1, 0]), i32([2, 1]), 3, 0.1)
    d = R.rlgen_token_logprobs_backward(z.cuda(), tok, 1.0, lp.stats, dlp).cpu()
    assert (d[SEQ[0]] == 0).all() and torch.isfinite(d[11:]).all() and bool((d[11:20] != 0).any())
