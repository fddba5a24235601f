"""A few steps of online DPO on a small policy, from token ids to gradients, the way a learner runs them.

    python examples/dpo_step.py

The policy is an embedding, a normed layer with windowed attention (examples/windowed_layer.py), dropout on its branch, a last norm and
an LM head.  A step: the sequences of all prompts as packed rows, norms and attention forward, logits, token log-probs, the loss of the
pairs that the rewards choose with its gradient, and back through the same operators.  Products with weights are plain matrix products;
everything between them is the library's.  At the end the policy is asked for its likeliest next tokens.
"""
import math
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
for path in (os.path.dirname(HERE), HERE):
    if path not in sys.path:
        sys.path.insert(0, path)
import paper_2410_18252_amd.rlgen as R  # noqa: E402
from windowed_layer import Layer  # noqa: E402


class Policy:
    def __init__(self, vocab=1003, d=256, eps=1e-5, drop_p=0.1, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layer = Layer(d=d, n_q=4, n_kv=2, h=64, window=50, sinks=2, dtype=dtype, seed=seed)
        self.embed = torch.randn(vocab, d, generator=g, device="cuda").to(dtype)
        self.lm_head = (torch.randn(vocab, d, generator=g, device="cuda") / math.sqrt(d)).to(dtype)
        self.gain1, self.gain2 = torch.ones(d, device="cuda"), torch.ones(d, device="cuda")
        self.eps, self.drop_p = eps, drop_p

    def forward(self, tokens, row_starts, positions, max_len, rng=None):
        """Packed token ids [rows] -> logits [rows, vocab], and what backward needs.  The residual stream is kept in 32 bits; without rng nothing is
        dropped."""
        drop = 0.0 if rng is None else self.drop_p
        h0, y0 = R.rlgen_add_rms_norm(self.embed[tokens.long()], self.gain1, self.eps, h_dtype=torch.float32)
        branch, saved = self.layer.forward(y0, row_starts, positions, max_len)
        h1, y1 = R.rlgen_add_rms_norm(branch, self.gain2, self.eps, residual=h0, drop_p=drop, rng=rng)
        return y1 @ self.lm_head.T, (tokens, h0, saved, h1, y1, drop, rng)

    def backward(self, dlogits, saved):
        """Gradients of every parameter outside the layer, and of the layer's own."""
        tokens, h0, layer, h1, y1, drop, rng = saved
        dh1, dbranch, dgain2 = R.rlgen_add_rms_norm_backward(h1, self.gain2, self.eps, dlogits @ self.lm_head, drop_p=drop, rng=rng)
        grads = self.layer.backward(dbranch, layer)
        _, dx, dgain1 = R.rlgen_add_rms_norm_backward(h0, self.gain1, self.eps, grads.pop("x"), dh=dh1)
        dembed = torch.zeros_like(self.embed, dtype=torch.float32).index_add_(0, tokens.long(), dx.float())
        return grads | {"embed": dembed, "gain1": dgain1, "gain2": dgain2, "lm_head": dlogits.T.contiguous() @ y1}


def targets_of(tokens, lens, prompts):
    """The token that each row predicts; rows whose prediction lies in the prompt, and last rows, have none."""
    out = torch.roll(tokens, -1)
    at = 0
    for n, p in zip(lens, prompts):
        out[at:at + p - 1] = -1
        out[at + n - 1] = -1
        at += n
    return out


def loss_and_gradients(policy, tokens, targets, row_starts, positions, max_len, ref, pos, neg, k, beta, rng=None):
    """Mean DPO loss of the pairs, and the gradients of the policy."""
    logits, saved = policy.forward(tokens, row_starts, positions, max_len, rng)
    lp = R.rlgen_token_logprobs(logits, targets, entropy=False)
    loss, dlp = R.rlgen_dpo_pairs(lp.logprobs, ref, row_starts, pos, neg, k, beta, weight=1.0 / pos.numel())
    R.rlgen_token_logprobs_backward(logits, targets, 1.0, lp.stats, dlp, out=logits)           # the gradient takes the logits' place
    return loss.mean(), policy.backward(logits, saved)


def batch(vocab, B, k, lo, hi, prompt, seed=1):
    """B prompts with k completions each: (tokens, targets, row_starts, positions, longest, pos, neg)."""
    g = torch.Generator().manual_seed(seed)
    lens = (prompt + torch.randint(lo, hi + 1, (B * k,), generator=g)).tolist()
    tokens = torch.randint(0, vocab, (sum(lens),), generator=g).int()
    starts = torch.tensor([0] + lens).cumsum(0).int()
    for b in range(B):                                       # a prompt's sequences begin alike
        first = int(starts[b * k])
        for i in range(1, k):
            at = int(starts[b * k + i])
            tokens[at:at + prompt] = tokens[first:first + prompt]
    positions = torch.cat([torch.arange(n) for n in lens]).int()
    pos, neg = R.rlgen_select_pairs(torch.rand(B, k, generator=g).cuda())
    return tokens.cuda(), targets_of(tokens, lens, [prompt] * (B * k)).cuda(), starts.cuda(), positions.cuda(), max(lens), pos, neg


def main(steps=5, B=6, k=4, lo=3, hi=120, prompt=17, beta=0.1, rate=0.02, quiet=False):
    say = (lambda *a: None) if quiet else print
    policy = Policy()
    tokens, targets, starts, positions, longest, pos, neg = batch(policy.lm_head.shape[0], B, k, lo, hi, prompt)
    ref = R.rlgen_token_logprobs(policy.forward(tokens, starts, positions, longest)[0], targets, entropy=False).logprobs
    rng = torch.tensor([1234, 0], dtype=torch.int64, device="cuda")
    for step in range(steps):
        rng[1] = step                                        # a new mask for every step
        loss, grads = loss_and_gradients(policy, tokens, targets, starts, positions, longest, ref, pos, neg, k, beta, rng)
        say(f"step {step}: loss {float(loss):.4f}, " + ", ".join(f"|{n}| {float(v.float().norm()):.2e}" for n, v in grads.items()))
        for name, grad in grads.items():
            owner = policy if hasattr(policy, name) else policy.layer
            p = getattr(owner, name)
            setattr(owner, name, (p.float() - rate * grad.float()).to(p.dtype))
    logits, _ = policy.forward(tokens, starts, positions, longest)
    last = (starts[1:] - 1).long()
    likely = R.rlgen_token_logprobs(logits[last], n_top=5)
    say("likeliest next tokens of the first sequence: " + ", ".join(f"{t} ({math.exp(p):.3f})" for t, p in zip(likely.top_tokens[0].tolist(), likely.top_logprobs[0].tolist())))
    return float(loss), grads, likely


if __name__ == "__main__":
    main()
