"""The gradients of examples/dpo_step.py's bf16 matrices against differences of its loss, between two places whose distance is known exactly: chosen elements move
by whole steps of their type, so that every one of them moves."""
import importlib.util
import os

import pytest
import torch

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("dpo_step", os.path.join(ROOT, "examples", "dpo_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def step_of(p):
    """bf16's step at a value: 2^-7 of the power of two below it."""
    return torch.exp2(torch.floor(torch.log2(p.float().abs().clamp(min=2.0 ** -100))) - 7)


@pytest.mark.parametrize("choice", [5, 6])
@pytest.mark.parametrize("name", ["lm_head", "embed"])
def test_gradients_of_matrices_are_slopes(example, name, choice):
    """Rounding: bf16 logits are rounded to 2^-8 of their size (about 1), a log-prob is off by about that, the loss of a pair by beta times the root of the summed
    rows times it, the mean of 8 independent pairs by a root of 8 less; four times as much at most.  A random choice of elements moves along
    the gradient's sign until the gradient calls for 24 times that between the two places: the response has to be there to a fifth, 2 of the 24 for
    rounding and a tenth for the loss's cube."""
    policy = example.Policy(drop_p=0.1)
    tokens, targets, starts, positions, longest, pos, neg = example.batch(1003, 8, 2, 40, 120, 9)
    rng = torch.tensor([7, 7], dtype=torch.int64, device="cuda")
    ref = R.rlgen_token_logprobs(example.Policy(seed=3).forward(tokens, starts, positions, longest)[0], targets, entropy=False).logprobs
    args = (tokens, targets, starts, positions, longest, ref, pos, neg, 2, 0.1, rng)
    grad, before = example.loss_and_gradients(policy, *args)[1][name].double(), getattr(policy, name)
    noise = 4 * 0.1 * (2 * 130) ** 0.5 * 2.0 ** -8 / 8 ** 0.5
    each = 2 * 4 * step_of(before).double() * grad.abs()                # four steps each way
    order = torch.randperm(each.numel(), generator=torch.Generator().manual_seed(choice)).cuda()
    gains = each.flatten()[order].cumsum(0)
    enough = int((gains < 24 * noise).sum()) + 1
    assert enough < order.numel()
    moves = torch.zeros_like(grad).flatten()
    moves[order[:enough]] = 1.0
    move = (moves.view_as(grad) * grad.sign() * 4 * step_of(before).double()).float()
    places = [(before.float() + move).to(before.dtype), (before.float() - move).to(before.dtype)]
    want = float(((places[0].double() - places[1].double()) * grad).sum())
    assert 20 * noise <= want <= 30 * noise                      # (all moved: a step across a power of two is rounded by half of itself at most)
    values = []
    for place in places:
        setattr(policy, name, place)
        values.append(float(example.loss_and_gradients(policy, *args)[0]))
    setattr(policy, name, before)
    assert abs(values[0] - values[1] - want) <= 0.1 * want + 2 * noise, (values, want, noise)
