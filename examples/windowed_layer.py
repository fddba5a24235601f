"""One attention layer with per-head norms and a sliding window, as a policy's layer is served and trained.

    python examples/windowed_layer.py

Serving: prompts of different lengths enter a cache in pages, then every sequence decodes token by token; plans, cache writes and
attention follow each other on the device, the host only enqueues them.  Half of the sequences end early: their requests ask for no
new token and cost nothing.  Training: the same tokens as packed rows, forward and backward.  Serving and training compute the
same function, so their outputs are compared at the end.
"""
import math
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)
import paper_2410_18252_amd.rlgen as R  # noqa: E402


class Layer:
    """q/k/v projection, per-head norms with rotation, windowed attention with sinks, output projection.  The two projections are plain
    matrix products; everything between them is the library's."""

    def __init__(self, d=1024, n_q=16, n_kv=4, h=64, rotary=64, window=256, sinks=4, theta=1e4, max_pos=8192, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def mat(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") / math.sqrt(shape[1])).to(dtype)

        self.n_q, self.n_kv, self.h, self.window, self.sinks, self.eps, self.scale = n_q, n_kv, h, window, sinks, 1e-6, 1 / math.sqrt(h)
        self.w_qkv, self.w_out = mat((n_q + 2 * n_kv) * h, d), mat(d, n_q * h)
        self.q_gain = 1 + 0.1 * torch.randn(h, generator=g, device="cuda")
        self.k_gain = 1 + 0.1 * torch.randn(h, generator=g, device="cuda")
        self.rope = R.rlgen_rope_table(max_pos, rotary, theta)

    def serve(self, x, plan, pages, page_table, max_new, max_total):
        """x [rows, d]: the new tokens of a plan.  Their keys and values go into the cache; [rows, d] comes back."""
        q = R.rlgen_qk_norm_rope(x @ self.w_qkv.T, self.q_gain, self.k_gain, self.eps, self.rope, plan.positions, pages=pages, slots=plan.slots)
        out, _ = R.rlgen_window_attention_paged(q, pages, page_table, plan.row_starts, plan.total_lens, max_new, max_total, self.window, self.sinks,
                                                self.scale)
        return out.flatten(1) @ self.w_out.T

    def forward(self, x, row_starts, positions, max_len):
        """x [rows, d]: whole sequences, packed.  Returns [rows, d] and what backward needs."""
        qkv = x @ self.w_qkv.T
        q, k, v = R.rlgen_qk_norm_rope(qkv, self.q_gain, self.k_gain, self.eps, self.rope, positions, n_kv_heads=self.n_kv)
        out, lse = R.rlgen_window_attention(q, k, v, row_starts, max_len, self.window, self.sinks, self.scale)
        return out.flatten(1) @ self.w_out.T, (x, qkv, q, k, v, out, lse, row_starts, positions, max_len)

    def backward(self, dy, saved):
        """Gradients of x and of every parameter, from that of the output."""
        x, qkv, q, k, v, out, lse, row_starts, positions, max_len = saved
        dout = (dy @ self.w_out).view_as(out)
        dq, dk, dv = R.rlgen_window_attention_backward(q, k, v, out, lse, dout, row_starts, max_len, self.window, self.sinks, self.scale)
        dqkv, dq_gain, dk_gain = R.rlgen_qk_norm_rope_backward(qkv, self.q_gain, self.k_gain, self.eps, self.rope, positions, dq, dk, dv)
        return {"x": dqkv @ self.w_qkv, "w_qkv": dqkv.T.contiguous() @ x, "w_out": dy.T.contiguous() @ out.flatten(1), "q_gain": dq_gain, "k_gain": dk_gain}


def main(S=24, lo=5, hi=900, steps=40, page=16, quiet=False):
    say = (lambda *a: None) if quiet else print
    layer = Layer()
    d, dtype = layer.w_out.shape[0], layer.w_out.dtype
    g = torch.Generator().manual_seed(1)
    prompt = torch.randint(lo, hi + 1, (S,), generator=g).tolist()
    ends = [n + (steps if i % 2 else steps // 2) for i, n in enumerate(prompt)]          # tokens of each sequence when it ends
    x = [torch.randn(n, d, generator=g).to(dtype).cuda() for n in ends]                   # what the layers below would hand over
    longest = max(prompt) + steps
    width = -(-longest // page)
    n_pages = sum(-(-n // page) for n in ends)
    free = torch.randperm(n_pages, generator=g).int().cuda()
    table = torch.full((S, width), -1, dtype=torch.int32, device="cuda")
    pages = torch.empty(n_pages, 2, layer.n_kv, page, layer.h, dtype=dtype, device="cuda")

    # serving: the prompts in one pass, then one token of each live sequence at a time
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    plan = R.rlgen_plan_pages(lens, torch.tensor(prompt, dtype=torch.int32, device="cuda"), page, free, table, sum(prompt))
    served = [[y] for y in layer.serve(torch.cat([t[:n] for t, n in zip(x, prompt)]), plan, pages, table, max(prompt), longest).split(prompt)]
    torch.cuda.synchronize()
    begun = time.perf_counter()
    for step in range(steps):
        live = [i for i in range(S) if prompt[i] + step < ends[i]]
        if not live:
            break
        new = torch.zeros(S, dtype=torch.int32)
        new[live] = 1
        plan = R.rlgen_plan_pages(plan.total_lens, new.cuda(), page, free, table, len(live), free_head=plan.counts[1:2])
        rows = torch.stack([x[i][prompt[i] + step] for i in live])
        for i, y in zip(live, layer.serve(rows, plan, pages, table, 1, longest)):
            served[i].append(y[None])
    torch.cuda.synchronize()
    rows, taken, total, faults = plan.counts.tolist()
    assert faults == 0 and taken == n_pages and plan.total_lens.tolist() == ends
    say(f"served {S} sequences: prompts of {min(prompt)} to {max(prompt)} tokens, {steps} steps in {1e3 * (time.perf_counter() - begun):.1f} ms, {taken} pages")

    # training: the same tokens at once
    starts = torch.tensor([0] + ends).cumsum(0).int().cuda()
    positions = torch.cat([torch.arange(n) for n in ends]).int().cuda()
    y, saved = layer.forward(torch.cat(x), starts, positions, max(ends))
    grads = layer.backward(torch.randn_like(y), saved)
    torch.cuda.synchronize()
    together = torch.cat([torch.cat(t) for t in served])
    far = float((together.float() - y.float()).norm() / y.float().norm())
    say(f"serving against training: relative difference {far:.1e}; gradients: " + ", ".join(f"|{k}| {float(v.float().norm()):.3g}" for k, v in grads.items()))
    assert all(torch.isfinite(v).all() for v in grads.values())
    return far, grads


if __name__ == "__main__":
    main()
