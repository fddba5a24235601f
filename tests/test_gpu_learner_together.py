"""The learner's operators together: norm with dropout, logits, log-probs, the pairs' loss and back, against 64-bit autograd; and as
examples/dpo_step.py runs them."""
import importlib.util
import os

import pytest
import torch

import learner_reference as L

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("drop, T", [(0.0, 1.0), (0.2, 0.7)])
def test_from_rows_to_gradients(drop, T):
    """All in 32 bits.  Every gradient is behind two products in a row with sums of 96 (logits), 501 (back through them) and 230 terms (weights),
    in all under 1000; a sum of n terms of random signs is off by n U of their magnitudes, which are about sqrt(n) times the sum: 1000 * 32 * 2^-24 of
    the gradient's size."""
    lens, k, d, V, eps = [30, 41, 60, 20, 3, 76], 3, 96, 501, 1e-5
    rows, starts = sum(lens), [0] + torch.tensor(lens).cumsum(0).tolist()
    g = torch.Generator().manual_seed(5)
    x, r, gain, W = (torch.randn(*s, generator=g) for s in ((rows, d), (rows, d), (d,), (V, d)))
    W = W / 5
    tokens = torch.randint(0, V, (rows,), generator=g)
    tokens[::5] = -1
    ref = torch.where(tokens >= 0, -torch.rand(rows, generator=g) * 6, 0.0)
    pos, neg, beta = [2, 0], [1, 1], 0.1
    rng = torch.tensor([3, 4], dtype=torch.int64, device="cuda")

    h, y = R.rlgen_add_rms_norm(x.cuda(), gain.cuda(), eps, residual=r.cuda(), drop_p=drop, rng=rng)
    logits = y @ W.cuda().T
    tok = tokens.int().cuda()
    lp = R.rlgen_token_logprobs(logits, tok, T)
    loss, dlp = R.rlgen_dpo_pairs(lp.logprobs, ref.cuda(), torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor(pos, dtype=torch.int32).cuda(),
                                  torch.tensor(neg, dtype=torch.int32).cuda(), k, beta, weight=0.5)
    dent = torch.full((rows,), -1e-3, device="cuda")                                # an entropy bonus beside the loss
    dz = R.rlgen_token_logprobs_backward(logits, tok, T, lp.stats, dlp, lp.entropy, dent, out=logits)
    dr, dx, dgain = R.rlgen_add_rms_norm_backward(h, gain.cuda(), eps, dz @ W.cuda(), drop_p=drop, rng=rng)
    dW = dz.T.contiguous() @ y

    leaves = [t.double().requires_grad_() for t in (x, r, gain, W)]
    f = L.keep_factors(rows, d, drop, 3, 4) if drop else 1.0
    _, y64, _ = L.add_norm(leaves[0], leaves[1], f, leaves[2], eps)
    all_lp = torch.log_softmax(y64 @ leaves[3].T / T, -1)
    live = tokens >= 0
    lp64 = torch.where(live, all_lp[torch.arange(rows), tokens.clamp(min=0)], 0.0)
    moved = lp64 - ref.double()
    sums = torch.stack([moved[a:b].sum() for a, b in zip(starts, starts[1:])]).view(2, k)
    losses = -torch.nn.functional.logsigmoid(beta * torch.stack([sums[b, pos[b]] - sums[b, neg[b]] for b in range(2)]))
    entropy = torch.where(live, -(all_lp.exp() * all_lp).sum(-1), 0.0)
    want = torch.autograd.grad(0.5 * losses.sum() - 1e-3 * entropy.sum(), leaves)
    assert float((loss.double().cpu() - losses.detach()).abs().max()) <= 1e-4
    for name, got, w in zip(("x", "residual", "gain", "W"), (dx, dr, dgain, dW), want):
        assert float((got.double().cpu() - w).norm()) <= 1000 * 32 * 2.0 ** -24 * float(w.norm()), name


def test_calls_on_two_streams_at_once():
    """Each stream's calls, parted rows and a two-launch gradient among them, give what they give alone."""
    def work(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        z, x = torch.randn(5, 90001, generator=g, device="cuda").bfloat16(), torch.randn(700, 1032, generator=g, device="cuda").bfloat16()
        tok, gain = torch.arange(5, dtype=torch.int32, device="cuda"), torch.randn(1032, generator=g, device="cuda")
        rng = torch.tensor([seed, 1], dtype=torch.int64, device="cuda")

        def run():
            r = R.rlgen_token_logprobs(z, tok, 0.7, n_top=9)
            d = R.rlgen_token_logprobs_backward(z, tok, 0.7, r.stats, r.entropy)
            h, y = R.rlgen_add_rms_norm(x, gain, 1e-5, drop_p=0.3, rng=rng)
            return [*r, d, h, y, *R.rlgen_add_rms_norm_backward(h, gain, 1e-5, y, drop_p=0.3, rng=rng)]
        return run

    runs = [work(1), work(2)]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(10):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i].append(runs[i]())
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for result in got[i] for a, b in zip(result, want[i]))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("dpo_step", os.path.join(ROOT, "examples", "dpo_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("B, k, lo, hi, prompt", [(6, 4, 3, 120, 17), (1, 2, 1, 1, 1)])
def test_the_example_runs(example, B, k, lo, hi, prompt):
    loss, grads, likely = example.main(2, B, k, lo, hi, prompt, quiet=True)
    assert loss == loss and all(torch.isfinite(v).all() for v in grads.values())
    assert set(grads) == {"embed", "gain1", "gain2", "lm_head", "w_qkv", "w_out", "q_gain", "k_gain"}
    assert (likely.top_logprobs[:, :-1] >= likely.top_logprobs[:, 1:]).all()


@pytest.mark.parametrize("name", ["gain1", "gain2", "lm_head", "embed"])
def test_the_examples_gradients_are_slopes(example, name):
    """The loss at two places along the gradient.  bf16 logits are rounded to 2^-8 of their size (about 1): a log-prob is off by about that, and the loss
    by beta times the root of the summed rows times it, four times as much at most; the step is ten times that each way.  What counts is the way between the two
    places as the parameters are rounded (many of a bf16 matrix do not move at all), times the gradient; the loss's square term falls out of the
    difference, and its cube is a tenth of it at most."""
    policy = example.Policy(drop_p=0.1)
    tokens, targets, starts, positions, longest, pos, neg = example.batch(1003, 8, 2, 40, 120, 9)
    rng = torch.tensor([7, 7], dtype=torch.int64, device="cuda")
    ref = R.rlgen_token_logprobs(example.Policy(seed=3).forward(tokens, starts, positions, longest)[0], targets, entropy=False).logprobs
    args = (tokens, targets, starts, positions, longest, ref, pos, neg, 2, 0.1, rng)
    _, grads = example.loss_and_gradients(policy, *args)
    grad, before = grads[name].float(), getattr(policy, name)
    size = float(grad.norm())
    noise = 4 * 0.1 * (2 * 130) ** 0.5 * 2.0 ** -8 / 8 ** 0.5
    t = 10 * noise / size                                    # a change of ten times the noise each way
    values, places = [], []
    for s in (t, -t):
        places.append((before.float() + s * grad / size).to(before.dtype))
        setattr(policy, name, places[-1])
        values.append(float(example.loss_and_gradients(policy, *args)[0]))
    setattr(policy, name, before)
    want = float(((places[0].double() - places[1].double()) * grad.double()).sum())
    assert want > 0 and abs(values[0] - values[1] - want) <= 0.1 * want + 2 * noise, (values, want, noise)
