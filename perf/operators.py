"""The paged cache's plan, the per-head norm with rotation and the windowed attention, as cases that can be timed and compared.

A case is one call of an operator: the plan of a pass over the paged cache (`plan`), the norms and rotation of queries and keys with the
cache write (`rope`) and their gradients (`rope_grad`), attention over packed sequences (`rows`), the same with its gradients
(`train`), a chunk of new tokens over the paged cache (`chunk`) and single tokens over it (`decode`).  Head layouts are those of the
models the framework runs and some generic ones.  The plain forms are elementary torch operations in 32 bits over padded batches.
"""
import math
import random

import numpy as np
import torch

own = False

# name: (query heads, kv heads, head dim, rotary dims, theta)
HEADS = {
    "tiny": (4, 4, 32, 8, 1e4),
    "g64": (16, 4, 64, 32, 1e4),
    "2.8b": (32, 32, 80, 20, 1e4),
    "g96": (12, 2, 96, 96, 1e4),
    "8b": (32, 8, 128, 128, 5e5),
    "1b": (8, 8, 256, 64, 1e4),
}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


def _case(name, op, heads, S, lo, hi, new=0, window=0, sinks=0, page=16, dtype="bf16", src="bf16"):
    return {"name": name, "op": op, "heads": heads, "S": S, "lo": lo, "hi": hi, "new": new, "window": window, "sinks": sinks,
            "page": page, "dtype": dtype, "src": src}


def listed():
    """lo..hi: tokens of a sequence before the pass (plan, rope), or in all (the others); new: tokens that the pass adds to it, where that
    is one number (0: the whole sequence is new)."""
    return [
        # a decode step's bookkeeping: 1000 requests of the chatbot workload add one token each
        _case("plan-decode-1000", "plan", "8b", 1000, 256, 1535, new=1),
        # the prompts of a whole batch arrive at once
        _case("plan-prompts-512", "plan", "2.8b", 512, 256, 512, page=32),
        # a decode step of 128 requests: one row each
        _case("rope-decode-128", "rope", "8b", 128, 256, 1535, new=1),
        # a prompt pass with the fp16 formats, part of each head rotated, heads whose rotary half is no multiple of eight
        _case("rope-prompts-2.8b", "rope", "2.8b", 21, 256, 512, dtype="f16", src="f16"),
        # the learner's backward pass over 16 sequences of about 500 tokens
        _case("rope-grad-8b", "rope_grad", "8b", 16, 257, 768),
        # a learner's forward pass over short and ragged sequences, from a single token on
        _case("rows-g64-short", "rows", "g64", 48, 1, 512, window=128, sinks=4, dtype="f16"),
        # a long prompt handled in chunks: 500 new tokens on each of six contexts
        _case("chunk-8b", "chunk", "8b", 6, 1000, 8000, new=500, window=1024, sinks=4),
        # training on long windowed sequences, grouped heads
        _case("train-8b-window", "train", "8b", 3, 1500, 4000, window=1024, sinks=4),
        # training on the summarisation workload's sequences, every earlier key visible
        _case("train-2.8b", "train", "2.8b", 24, 257, 576, dtype="f16"),
        # one conversation of 32000 tokens, every key visible: few rows, a long axis
        _case("decode-8b-1", "decode", "8b", 1, 32001, 32001, new=1),
        # a serving batch of windowed layers, long contexts of which the window and the sinks are read
        _case("decode-8b-64-window", "decode", "8b", 64, 1, 9000, new=1, window=1024, sinks=4, page=32),
        # the summarisation workload's decode step
        _case("decode-2.8b-512", "decode", "2.8b", 512, 257, 576, new=1, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# seconds of a pass at 3 TB/s and 0.3 PFLOP/s
def _seconds(case):
    w = work(case)
    return w["bytes"] / 3e12 + w["flops"] / 3e14 + 5e-6


def _fits(case):
    """The padded plain form's scores in 32 bits, and the cache, stay small beside the card's memory."""
    hq, hkv, h, _, _ = HEADS[case["heads"]]
    q = case["new"] or case["hi"]
    scores = 4.0 * case["S"] * hq * q * case["hi"] if case["op"] in ("rows", "train", "chunk") else 0.0
    return scores <= 8e9 and 4.0 * hkv * h * case["S"] * case["hi"] <= 8e9 and 3072 not in case.values()


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        op = rng.choice(["plan", "rope", "rope_grad", "rows", "chunk", "train", "train", "decode", "decode"])
        heads = rng.choice(list(HEADS))
        window = rng.choice([0, _log_int(rng, 1, 4096)])
        sinks = rng.choice([0, 1, 4, rng.randint(1, 100)]) if window else 0
        page = rng.choice([8, 16, 16, 32, 64])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        S = _log_int(rng, 1, 512)
        if op == "plan":
            lo = rng.randint(0, 700)
            c = _case("", op, heads, _log_int(rng, 1, 4000), lo, lo + _log_int(rng, 1, 1500), new=rng.choice([0, 1, 1, rng.randint(2, 40)]), page=page)
        elif op in ("rope", "rope_grad"):
            new = rng.choice([0, 1]) if op == "rope" else 0
            c = _case("", op, heads, S if new else _log_int(rng, 1, 32), rng.randint(1, 256), rng.randint(257, 1200), new=new, page=page, dtype=dtype,
                      src=rng.choice([dtype, "f32"]))
        elif op in ("rows", "train"):
            hi = _log_int(rng, 1, 4096)
            c = _case("", op, heads, _log_int(rng, 1, 64), rng.randint(1, hi), hi, window=window, sinks=sinks, dtype=dtype)
        elif op == "chunk":
            new = _log_int(rng, 2, 700)
            hi = new + _log_int(rng, 1, 12000)
            c = _case("", op, heads, _log_int(rng, 1, 16), rng.randint(new, hi), hi, new=new, window=window, sinks=sinks, page=page, dtype=dtype)
        else:
            hi = _log_int(rng, 1, 40000)
            c = _case("", op, heads, S, rng.randint(1, hi), hi, new=1, window=window, sinks=sinks, page=page, dtype=dtype)
        del c["name"]
        if _seconds(c) <= 0.9 * most and _fits(c):
            return c


# ------------------------------------------------------------------------------------------------ lengths and necessary work


def _lens(case):
    """One length for each sequence, spread evenly over lo..hi."""
    S, lo, hi = case["S"], case["lo"], case["hi"]
    return [hi] if S == 1 else [lo + (hi - lo) * i // (S - 1) for i in range(S)]


def _ctx_new(case, order):
    """(tokens in the cache before the pass, tokens that it adds) of each sequence, in the order given."""
    lens = [_lens(case)[i] for i in order]
    if case["op"] in ("plan", "rope", "rope_grad"):
        return ([0] * len(lens), lens) if case["new"] == 0 else (lens, [case["new"]] * len(lens))
    if case["new"] == 0:
        return [0] * len(lens), lens
    return [n - case["new"] for n in lens], [case["new"]] * len(lens)


def _visible(case, ctx, new):
    """Visible pairs of one sequence, and how many of its keys any of its queries sees."""
    p = np.arange(ctx, ctx + new, dtype=np.int64)
    W, sinks = case["window"], case["sinks"]
    if W == 0:
        return int((p + 1).sum()), ctx + new
    first = np.maximum(p - W + 1, 0)
    low = max(ctx - W + 1, 0)
    return int((p + 1 - first + np.minimum(first, sinks)).sum()), ctx + new - low + min(low, sinks)


def work(case):
    hq, hkv, h, r, _ = HEADS[case["heads"]]
    ctx, new = _ctx_new(case, range(case["S"]))
    S, rows, P = case["S"], sum(new), case["page"]
    if case["op"] == "plan":
        # plain counting: every length, page and row once
        had = sum(-(-c // P) for c in ctx)
        need = sum(-(-(c + n) // P) for c, n in zip(ctx, new))
        return {"bytes": 4.0 * (2 * S + 2 * (need - had) + 2 * S + 2 * rows), "flops": 0.0}
    e, se = 2.0, 4.0 if case["src"] == "f32" else 2.0
    width = (hq + 2 * hkv) * h
    if case["op"] == "rope":
        return {"bytes": rows * (width * (se + e) + 8.0) + 4.0 * r * min(rows, max(c + n for c, n in zip(ctx, new))), "flops": 6.0 * rows * width}
    if case["op"] == "rope_grad":
        return {"bytes": rows * ((hq + hkv) * h * (2 * se + e) + hkv * h * (se + e) + 4.0) + 4.0 * r * max(new), "flops": 14.0 * rows * width}
    pairs = keys = 0
    for c, n in zip(ctx, new):
        a, b = _visible(case, c, n)
        pairs, keys = pairs + a, keys + b
    forward = {"bytes": e * h * (2 * rows * hq + 2 * keys * hkv) + 4.0 * rows * hq, "flops": 4.0 * h * hq * pairs}
    if case["op"] == "train":
        return {"bytes": forward["bytes"] + e * h * (4 * rows * hq + 4 * rows * hkv), "flops": 14.0 * h * hq * pairs}
    return forward


# ------------------------------------------------------------------------------------------------ inputs


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _gen(seed):
    return torch.Generator(device=_device()).manual_seed(int(seed) * 1000003 + 29)


def _normal(g, *shape, dtype, scale=1.0):
    t = torch.empty(*shape, dtype=dtype if dtype != torch.float16 else torch.float32, device=_device()).normal_(0.0, scale, generator=g)
    return t.to(dtype)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=_device())


def _tables(case, seed, ctx, total, spare=8):
    """A page table with the pages of the contexts at random places, and the pages left, as a cache that has run for a while has them."""
    P = case["page"]
    rng = np.random.default_rng(int(seed) * 7 + 3)
    need = sum(-(-t // P) for t in total)
    n_pages = need + spare
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((case["S"], max(1, -(-max(total) // P)) + 1), -1, np.int32)
    have = -(-np.asarray(ctx) // P)
    col = np.arange(table.shape[1])[None, :] < have[:, None]
    table[col] = ids[: int(have.sum())]
    return torch.from_numpy(table).to(_device()), torch.from_numpy(ids[int(have.sum()):].copy()).to(_device()), n_pages


def prepare(case, seed):
    hq, hkv, h, r, theta = HEADS[case["heads"]]
    dev, g, dt = _device(), _gen(seed), TYPES[case["dtype"]]
    order = list(range(case["S"]))
    random.Random(seed).shuffle(order)
    ctx, new = _ctx_new(case, order)
    total = [c + n for c, n in zip(ctx, new)]
    rows, op = sum(new), case["op"]
    s = {"case": case, "rows": rows, "max_new": max(new), "max_total": max(total), "scale": 1.0 / math.sqrt(h)}
    starts = np.concatenate([[0], np.cumsum(new)])
    s["row_starts"] = _i32(starts.tolist())
    s["total_lens"] = _i32(total)
    if op == "plan":
        s["ctx_lens"], s["new_lens"] = _i32(ctx), _i32(new)
        s["table"], s["free"], _ = _tables(case, seed, ctx, total)
        s["out"] = (torch.empty(len(ctx), dtype=torch.int32, device=dev), torch.empty(len(ctx) + 1, dtype=torch.int32, device=dev),
                    torch.empty(rows, dtype=torch.int32, device=dev), torch.empty(rows, dtype=torch.int32, device=dev),
                    torch.empty(4, dtype=torch.int32, device=dev))
        return s
    if op in ("rope", "rope_grad"):
        pos = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)])
        ang = np.arange(max(total))[:, None] * theta ** (-2.0 * np.arange(r // 2)[None, :] / r)
        s["rope"] = torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)).to(dev)
        s["positions"] = _i32(pos.tolist())
        s["qkv"] = _normal(g, rows, (hq + 2 * hkv) * h, dtype=TYPES[case["src"]], scale=1.5)
        s["q_gain"] = 1.0 + _normal(g, h, dtype=torch.float32, scale=0.1)
        s["k_gain"] = 1.0 + _normal(g, h, dtype=torch.float32, scale=0.1)
        if op == "rope":
            P = case["page"]
            n_pages = sum(-(-n // P) for n in new) + 8 if case["new"] == 0 else case["S"] + 8
            ids = np.random.default_rng(int(seed) * 7 + 3).permutation(n_pages)
            # the pages that this pass writes: a whole sequence's from its first token on, or the last page of each
            first = np.concatenate([[0], np.cumsum([(-(-n // P)) if case["new"] == 0 else 1 for n in new])])
            place = np.concatenate([ids[first[i] + (np.arange(n) // P if case["new"] == 0 else np.zeros(n, np.int64))] * P + (np.arange(c, c + n) % P)
                                    for i, (c, n) in enumerate(zip(ctx, new))])
            s["slots"] = _i32(place.tolist())
            s["pages"] = torch.zeros(n_pages, 2, hkv, P, h, dtype=dt, device=dev)
            s["out"] = torch.empty(rows, hq, h, dtype=dt, device=dev)
        else:
            s["dq"], s["dk"], s["dv"] = (_normal(g, rows, n, h, dtype=dt, scale=0.1) for n in (hq, hkv, hkv))
        return s
    s["q"] = _normal(g, rows, hq, h, dtype=dt)
    if op in ("rows", "train"):
        s["k"], s["v"] = _normal(g, rows, hkv, h, dtype=dt), _normal(g, rows, hkv, h, dtype=dt)
        if op == "train":
            s["do"] = _normal(g, rows, hq, h, dtype=dt)
        return s
    s["table"], _, n_pages = _tables(case, seed, total, total)
    s["pages"] = _normal(g, n_pages, 2, hkv, case["page"], h, dtype=dt)
    s["out"] = torch.empty(rows, hq, h, dtype=dt, device=dev), torch.empty(rows, hq, dtype=torch.float32, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ plain forms


def _plain_plan(s):
    P, table, free = s["case"]["page"], s["table"], s["free"]
    ctx, new = s["ctx_lens"].long(), s["new_lens"].long()
    total = ctx + new
    had, need = (ctx + P - 1) // P, (total + P - 1) // P
    take = need - had
    ends = torch.cumsum(new, 0)
    starts = torch.cat([ends.new_zeros(1), ends])
    first = torch.cumsum(take, 0) - take
    col = torch.arange(table.shape[1], device=table.device)[None, :]
    at = first[:, None] + col - had[:, None]
    fresh = (col >= had[:, None]) & (col < need[:, None])
    table.copy_(torch.where(fresh, free[at.clamp(0, free.numel() - 1)], table))
    r = torch.arange(s["rows"], device=table.device)
    seq = torch.searchsorted(ends, r, right=True)
    pos = ctx[seq] + r - starts[seq]
    slots = table[seq, pos // P].long() * P + pos % P
    counts = torch.stack([ends[-1], take.sum(), total.max(), torch.zeros_like(ends[-1])])
    return [table] + [x.to(torch.int32) for x in (total, starts, slots, pos, counts)]


def _rotate(y, rope, r):
    a, b = y[..., : r // 2], y[..., r // 2: r]
    c, t = rope[:, None, :, 0], rope[:, None, :, 1]
    return torch.cat([a * c - b * t, b * c + a * t, y[..., r:]], -1)


def _plain_rope(s):
    hq, hkv, h, r, _ = HEADS[s["case"]["heads"]]
    P, pages = s["case"]["page"], s["pages"]
    x = s["qkv"].float().view(s["rows"], hq + 2 * hkv, h)
    rope = s["rope"][s["positions"].long()]
    gain = torch.cat([s["q_gain"].expand(hq, h), s["k_gain"].expand(hkv, h)])
    y = x[:, : hq + hkv]
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * gain
    y = _rotate(y, rope, r).to(pages.dtype)
    slot = s["slots"].long()
    pages[slot // P, 0, :, slot % P] = y[:, hq:]
    pages[slot // P, 1, :, slot % P] = x[:, hq + hkv:].to(pages.dtype)
    return [y[:, :hq], pages]


def _plain_rope_grad(s):
    hq, hkv, h, r, _ = HEADS[s["case"]["heads"]]
    x = s["qkv"].float().view(s["rows"], hq + 2 * hkv, h)[:, : hq + hkv]
    rope = s["rope"][s["positions"].long()]
    back = torch.stack([rope[..., 0], -rope[..., 1]], -1)
    gain = torch.cat([s["q_gain"].expand(hq, h), s["k_gain"].expand(hkv, h)])
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * rstd
    dy = _rotate(torch.cat([s["dq"], s["dk"]], 1).float(), back, r)
    dg = dy * n
    t = dy * gain
    dx = rstd * (t - n * (t * n).mean(-1, keepdim=True))
    dqkv = torch.cat([dx, s["dv"].float()], 1).to(s["qkv"].dtype).view(s["rows"], -1)
    return [dqkv, dg[:, :hq].sum((0, 1)), dg[:, hq:].sum((0, 1))]


def _row_index(s):
    """(sequence, place in it) of every row."""
    starts = s["row_starts"].long()
    r = torch.arange(s["rows"], device=starts.device)
    seq = torch.searchsorted(starts[1:].contiguous(), r, right=True)
    return seq, r - starts[seq]


def _pad(x, s, seq, at):
    out = x.new_zeros((s["case"]["S"], s["max_new"]) + x.shape[1:], dtype=torch.float32)
    out[seq, at] = x.float()
    return out


def _grouped(x, hkv):
    """[S, L, heads, h] -> [S, kv heads, heads of the group * L, h]"""
    S, L, n, h = x.shape
    return x.view(S, L, hkv, n // hkv, h).permute(0, 2, 3, 1, 4).reshape(S, hkv, -1, h)


def _ungrouped(x, L):
    """[S, kv heads, heads of the group * L, ...] -> [S, L, heads, ...]"""
    S, hkv, gl = x.shape[:3]
    x = x.view((S, hkv, gl // L, L) + x.shape[3:])
    x = x.permute((0, 3, 1, 2) + tuple(range(4, x.dim())))
    return x.reshape((S, L, hkv * (gl // L)) + x.shape[4:])


def _plain_scores(s, q, k, pos_q, pos_k, live):
    """Masked scores of padded queries against keys; pos_q [S, L], pos_k and live [S, T]."""
    W, sinks = s["case"]["window"], s["case"]["sinks"]
    seen = (pos_k[:, None, :] <= pos_q[:, :, None]) & live[:, None, :]
    if W:
        seen = seen & ((pos_k[:, None, :] > pos_q[:, :, None] - W) | (pos_k[:, None, :] < sinks))
    sc = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    S, hkv, gl, T = sc.shape
    L = pos_q.shape[1]
    return sc.view(S, hkv, gl // L, L, T).masked_fill(~seen[:, None, None], float("-inf")).view(S, hkv, gl, T)


def _plain_softmax(sc):
    """Probabilities and log-sum-exp; a row that sees nothing has zeros and -inf."""
    m = sc.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    e = torch.exp(sc - m)
    z = e.sum(-1, keepdim=True)
    return e / torch.where(z > 0, z, torch.ones_like(z)), (torch.log(z) + m)[..., 0]


def _plain_rows(s, grad):
    hkv = HEADS[s["case"]["heads"]][1]
    dt = s["q"].dtype
    seq, at = _row_index(s)
    L = s["max_new"]
    q = _grouped(_pad(s["q"], s, seq, at), hkv)
    k, v = (_pad(s[n], s, seq, at).transpose(1, 2).contiguous() for n in ("k", "v"))
    pos = torch.arange(L, device=q.device)[None, :].expand(s["case"]["S"], L)
    live = pos < s["total_lens"].long()[:, None]
    p, lse = _plain_softmax(_plain_scores(s, q, k, pos, pos, live))
    o = torch.matmul(p, v)
    got = [_ungrouped(o, L)[seq, at].to(dt), _ungrouped(lse, L)[seq, at]]
    if not grad:
        return got
    do = _grouped(_pad(s["do"], s, seq, at), hkv)
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = torch.matmul(do, v.transpose(-1, -2))
    ds = p * (ds - (do * o).sum(-1, keepdim=True))
    dq = torch.matmul(ds, k) * s["scale"]
    dk = torch.matmul(ds.transpose(-1, -2), q) * s["scale"]
    return got + [_ungrouped(dq, L)[seq, at].to(dt), dk.transpose(1, 2)[seq, at].to(dt), dv.transpose(1, 2)[seq, at].to(dt)]


def _plain_paged(s):
    hkv = HEADS[s["case"]["heads"]][1]
    P, W, sinks = s["case"]["page"], s["case"]["window"], s["case"]["sinks"]
    seq, at = _row_index(s)
    L = s["max_new"]
    total = s["total_lens"].long()
    pos_q = (total - (s["row_starts"][1:] - s["row_starts"][:-1]))[:, None] + torch.arange(L, device=total.device)[None, :]
    T = s["max_total"]
    c = torch.arange(min(T, sinks + W + L - 1) if W else T, device=total.device)[None, :]
    # the sinks' columns, then the window's
    pos_k = torch.where(c < sinks, c, (pos_q[:, :1] - W + 1).clamp(min=sinks) + c - sinks) if W else c.expand(s["case"]["S"], T)
    live = pos_k < total[:, None]
    pos_k = torch.minimum(pos_k, total[:, None] - 1)
    page = s["table"].long().gather(1, pos_k // P)
    k, v = (s["pages"][page, i, :, pos_k % P].float().transpose(1, 2).contiguous() for i in (0, 1))
    q = _grouped(_pad(s["q"], s, seq, at), hkv)
    p, lse = _plain_softmax(_plain_scores(s, q, k, pos_q, pos_k, live))
    return [_ungrouped(torch.matmul(p, v), L)[seq, at].to(s["q"].dtype), _ungrouped(lse, L)[seq, at]]


# ------------------------------------------------------------------------------------------------ one pass


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "plan":
            return _plain_plan(s)
        if op == "rope":
            return _plain_rope(s)
        if op == "rope_grad":
            return _plain_rope_grad(s)
        return _plain_rows(s, op == "train") if op in ("rows", "train") else _plain_paged(s)
    import paper_2410_18252_amd.rlgen as R
    if op == "plan":
        plan = R.rlgen_plan_pages(s["ctx_lens"], s["new_lens"], case["page"], s["free"], s["table"], s["rows"], out=s["out"])
        return [s["table"], *plan]
    if op == "rope":
        q = R.rlgen_qk_norm_rope(s["qkv"], s["q_gain"], s["k_gain"], EPS, s["rope"], s["positions"], pages=s["pages"], slots=s["slots"],
                                 out=s["out"])
        return [q, s["pages"]]
    if op == "rope_grad":
        return list(R.rlgen_qk_norm_rope_backward(s["qkv"], s["q_gain"], s["k_gain"], EPS, s["rope"], s["positions"], s["dq"], s["dk"], s["dv"]))
    if op in ("rows", "train"):
        out, lse = R.rlgen_window_attention(s["q"], s["k"], s["v"], s["row_starts"], s["max_new"], case["window"], case["sinks"], s["scale"])
        if op == "rows":
            return [out, lse]
        grads = R.rlgen_window_attention_backward(s["q"], s["k"], s["v"], out, lse, s["do"], s["row_starts"], s["max_new"], case["window"],
                                                  case["sinks"], s["scale"])
        return [out, lse, *grads]
    return list(R.rlgen_window_attention_paged(s["q"], s["pages"], s["table"], s["row_starts"], s["total_lens"], s["max_new"], s["max_total"],
                                               case["window"], case["sinks"], s["scale"], out=s["out"]))


# ------------------------------------------------------------------------------------------------ 64 bits


def _exact_heads(case, s):
    """Normalised and rotated heads in complex form: the rotation of a pair is a product with e^(i angle)."""
    hq, hkv, h, r, theta = HEADS[case["heads"]]
    x = s["qkv"].double().reshape(-1, hq + 2 * hkv, h)
    turn = torch.view_as_complex(s["rope"].double().contiguous())[s["positions"].long()][:, None, :]
    norm = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / h + EPS)
    return x, x / norm, norm, turn


def _turned(y, turn, r):
    z = torch.complex(y[..., : r // 2].contiguous(), y[..., r // 2: r].contiguous()) * turn
    return torch.cat([z.real, z.imag, y[..., r:]], -1)


def _exact_attention(case, scale, q, k, v, ctx, do=None):
    """One sequence: q [n, Hq, h] at positions ctx.., k and v [T, Hkv, h], all in 64 bits."""
    n, hq, h = q.shape
    T, hkv, _ = k.shape
    i, j = torch.arange(ctx, ctx + n, device=q.device)[:, None], torch.arange(T, device=q.device)[None, :]
    hidden = j > i
    if case["window"]:
        hidden |= (i - j >= case["window"]) & (j >= case["sinks"])
    out, lse, dq, dk, dv = torch.zeros_like(q), q.new_zeros(n, hq), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a in range(hq):
        b = a // (hq // hkv)
        z = (q[:, a] @ k[:, b].T * scale).masked_fill(hidden, float("-inf"))
        lse[:, a] = torch.logsumexp(z, -1)
        p = torch.exp(z - lse[:, a:a + 1])
        out[:, a] = p @ v[:, b]
        if do is not None:
            dv[:, b] += p.T @ do[:, a]
            w = do[:, a] @ v[:, b].T
            w = p * (w - (p * w).sum(-1, keepdim=True)) * scale
            dq[:, a] = w @ k[:, b]
            dk[:, b] += w.T @ q[:, a]
    return out, lse, dq, dk, dv


def exact(case, seed):
    op = case["op"]
    if op == "plan":
        return None
    hq, hkv, h, r, _ = HEADS[case["heads"]]
    s = prepare(case, seed)
    if op in ("rope", "rope_grad"):
        x, n, norm, turn = _exact_heads(case, s)
        gain = torch.cat([s["q_gain"].double().expand(hq, h), s["k_gain"].double().expand(hkv, h)])
        if op == "rope":
            y = _turned(n[:, : hq + hkv] * gain, turn, r)
            pages = s["pages"].double()
            P = case["page"]
            flat = pages.permute(0, 3, 1, 2, 4).reshape(-1, 2, hkv, h)
            flat[s["slots"].long()] = torch.stack([y[:, hq:], x[:, hq + hkv:]], 1)
            return [y[:, :hq], flat.view(-1, P, 2, hkv, h).permute(0, 2, 3, 1, 4).contiguous()]
        d = _turned(torch.cat([s["dq"], s["dk"]], 1).double(), turn.conj(), r)
        n, norm = n[:, : hq + hkv], norm[:, : hq + hkv]
        t = d * gain
        dx = (t - n * (t * n).sum(-1, keepdim=True) / h) / norm
        return [torch.cat([dx, s["dv"].double()], 1).reshape(s["rows"], -1), (d * n)[:, :hq].sum((0, 1)), (d * n)[:, hq:].sum((0, 1))]
    if 14.0 * work(case)["flops"] > 14e13 or case["S"] * hq > 40000:
        return None
    q = s["q"].double()
    starts, total = s["row_starts"].tolist(), s["total_lens"].tolist()
    got = [torch.zeros_like(q), q.new_zeros(q.shape[:2])]
    if op == "train":
        got += [torch.zeros_like(q), s["k"].double().zero_(), s["v"].double().zero_()]
    for i, t in enumerate(total):
        a, b = starts[i], starts[i + 1]
        if op in ("rows", "train"):
            k, v = s["k"][a:b].double(), s["v"][a:b].double()
        else:
            P = case["page"]
            pages = s["pages"][s["table"][i, : -(-t // P)].long()].double()
            k, v = pages.permute(1, 0, 3, 2, 4).reshape(2, -1, hkv, h)[:, :t]
        parts = _exact_attention(case, s["scale"], q[a:b], k, v, t - (b - a), s["do"][a:b].double() if op == "train" else None)
        for whole, part in zip(got, parts):
            whole[a:b] = part
    return got
