"""Norms with dropout and residual, token log-probs of logits and the pairs' loss, as cases that can be timed and compared.

A case is one call of an operator: the residual's addition with dropout and a root-mean-square norm (`norm`) and its gradients
(`norm_grad`), log-probs of given tokens with entropy and top alternatives (`logprobs`) and their gradient (`logprobs_grad`), the DPO loss of
packed sequences' pairs with its gradient (`dpo`).  Widths and vocabularies are those of the models the framework runs and generic
ones.  The plain forms are elementary torch operations in 32 bits; the generator of the dropout masks is integer arithmetic on both sides, and
sums over long sequences are taken in 64 bits.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2.0, "f16": 2.0, "f32": 4.0, "e4m3": 1.0}
EPS = 1e-5
BETA = 0.1


def _norm(name, op, rows, width, dtype="bf16", res="bf16", y="bf16", group=0, drop=0.0):
    """res: type of the residual stream; y: type of the norm's output; group: columns to a scale (e4m3; 0: the whole row)."""
    return {"name": name, "op": op, "rows": rows, "width": width, "dtype": dtype, "res": res, "y": y, "group": group, "drop": drop}


def _logits(name, op, rows, vocab, dtype="bf16", pad=0, top=0, temperature=0.7, skipped=0.0, entropy=True):
    """pad: elements between two rows; skipped: share of the rows that have no token (prompts, padding)."""
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "pad": pad, "top": top, "temperature": temperature,
            "skipped": skipped, "entropy": entropy}


def _dpo(name, B, k, lo, hi):
    """B prompts with k sequences each, of lo..hi rows."""
    return {"name": name, "op": "dpo", "B": B, "k": k, "lo": lo, "hi": hi}


def listed():
    return [
        # a serving step of 128 requests: residual, norm, and the input of an 8-bit product
        _norm("norm-decode-128", "norm", 128, 4096, y="e4m3"),
        # a prompt pass with the fp16 formats over a residual stream in 32 bits
        _norm("norm-2.8b-f16", "norm", 7001, 2560, dtype="f16", res="f32", y="f16"),
        # the learner's forward pass over 16 thousand packed rows, with dropout on the branch
        _norm("norm-drop-8b", "norm", 16384, 4096, drop=0.1),
        # the backward pass of a small batch at the 1B width, the residual stream in 32 bits
        _norm("norm-grad-1b", "norm_grad", 3001, 2048, dtype="f16", res="f32", y="f16"),
        # the learner's backward pass over 16 thousand packed rows
        _norm("norm-grad-drop-8b", "norm_grad", 16384, 4096, drop=0.1),
        # one request of a serving loop that asks for the alternatives of its token
        _logits("logprobs-1", "logprobs", 1, 50304, top=5),
        # a serving batch that asks for many, at a vocabulary whose rows start anywhere
        _logits("logprobs-300-odd", "logprobs", 300, 100003, dtype="f16", top=20),
        # the learner's rows at the 8B vocabulary; a quarter of them are prompts
        _logits("logprobs-8b", "logprobs", 8192, 128256, temperature=1.0, skipped=0.25),
        # gradients of log-probs and entropies in 32 bits, odd vocabulary
        _logits("logprobs-grad-odd", "logprobs_grad", 701, 50021, dtype="f32"),
        # the learner's gradient at the 8B vocabulary
        _logits("logprobs-grad-8b", "logprobs_grad", 8192, 128256, temperature=1.0, skipped=0.25, entropy=False),
        # the summarisation workload's pairs: 512 prompts, two completions each
        _dpo("dpo-512x2", 512, 2, 64, 576),
        # few prompts with four long completions each
        _dpo("dpo-16x4-long", 16, 4, 300, 9000),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# seconds of a pass at 3 TB/s
def _seconds(case):
    return work(case)["bytes"] / 3e12 + 5e-6


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "logprobs", "logprobs", "logprobs_grad", "logprobs_grad", "dpo"])
        if op in ("norm", "norm_grad"):
            dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
            width = rng.choice([128, 1024, 2048, 2560, 4096, 8 * _log_int(rng, 1, 2048), 8 * _log_int(rng, 1, 2048)])
            y = rng.choice([dtype, "e4m3"]) if op == "norm" else dtype
            c = _norm("", op, _log_int(rng, 1, 32768), width, dtype=dtype, res=rng.choice([dtype, "f32"]), y=y,
                      group=rng.choice([0, 32, 64, 128]) if y == "e4m3" else 0, drop=rng.choice([0.0, 0.1, rng.uniform(0.01, 0.6)]))
        elif op == "dpo":
            lo = rng.randint(1, 300)
            c = _dpo("", _log_int(rng, 1, 1024), rng.randint(2, 8), lo, lo + _log_int(rng, 1, 9000))
        else:
            vocab = rng.choice([1024, 50304, 128256, _log_int(rng, 70, 200000), _log_int(rng, 70, 200000)])
            c = _logits("", op, _log_int(rng, 1, 8192), vocab, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                        pad=rng.choice([0, 0, rng.randint(1, 70)]), top=rng.choice([0, 1, 5, 20, rng.randint(1, 64)]) if op == "logprobs" else 0,
                        temperature=rng.choice([0.7, 1.0, rng.uniform(0.3, 2.0)]), skipped=rng.choice([0.0, 0.3, rng.uniform(0.0, 0.9)]),
                        entropy=rng.choice([True, False]))
        del c["name"]
        if _seconds(c) <= 0.9 * most:
            return c


# ------------------------------------------------------------------------------------------------ necessary work


def _lens(case):
    """One length for each sequence, spread evenly over lo..hi."""
    n, lo, hi = case["B"] * case["k"], case["lo"], case["hi"]
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _skipped(case):
    return int(case["rows"] * case["skipped"])


def work(case):
    op = case["op"]
    if op == "dpo":
        rows, n = sum(_lens(case)), case["B"] * case["k"]
        return {"bytes": 12.0 * rows + 4.0 * (n + 1) + 12.0 * case["B"], "flops": 4.0 * rows}
    if op in ("logprobs", "logprobs_grad"):
        rows, V, e = case["rows"], case["vocab"], BYTES[case["dtype"]]
        live = rows - _skipped(case)
        if op == "logprobs":
            return {"bytes": live * V * e + rows * (12.0 + 4.0 + 4.0 * case["entropy"] + 8.0 * case["top"]), "flops": 7.0 * live * V}
        return {"bytes": (live + rows) * V * e + rows * (12.0 + 4.0 + 8.0 * case["entropy"]), "flops": 7.0 * live * V}
    n, d = case["rows"] * case["width"], case["width"]
    e, r, y = BYTES[case["dtype"]], BYTES[case["res"]], BYTES[case["y"]]
    scales = case["rows"] * -(-d // case["group"] if case["group"] else -1) * 4.0 if case["y"] == "e4m3" else 0.0
    if op == "norm":
        return {"bytes": n * (e + 2 * r + y) + 4.0 * d + scales, "flops": 7.0 * n}
    return {"bytes": n * (2 * e + 3 * r) + 8.0 * d, "flops": 13.0 * n}


# ------------------------------------------------------------------------------------------------ inputs


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _gen(seed):
    return torch.Generator(device=_device()).manual_seed(int(seed) * 1000003 + 57)


def _normal(g, *shape, dtype, scale=1.0):
    t = torch.empty(*shape, dtype=dtype if dtype != torch.float16 else torch.float32, device=_device()).normal_(0.0, scale, generator=g)
    return t.to(dtype)


def _uniform(g, *shape, lo=0.0, hi=1.0):
    return torch.empty(*shape, dtype=torch.float32, device=_device()).uniform_(lo, hi, generator=g)


def prepare(case, seed):
    dev, g, op = _device(), _gen(seed), case["op"]
    s = {"case": case}
    if op == "dpo":
        lens = _lens(case)
        random.Random(seed).shuffle(lens)
        rows, B, k = sum(lens), case["B"], case["k"]
        s["row_starts"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(dev)
        s["ref"] = -2.0 * _uniform(g, rows) ** 2
        # the policy has moved a little from the reference
        s["pol"] = s["ref"] + _normal(g, rows, dtype=torch.float32, scale=0.05)
        s["pos"] = torch.randint(0, k, (B,), dtype=torch.int32, device=dev, generator=g)
        s["neg"] = ((s["pos"] + 1 + torch.randint(0, k - 1, (B,), dtype=torch.int32, device=dev, generator=g)) % k).to(torch.int32)
        s["out"] = torch.empty(B, device=dev), torch.empty(rows, device=dev)
        return s
    dt, rows = TYPES[case["dtype"]], case["rows"]
    if op in ("logprobs", "logprobs_grad"):
        V = case["vocab"]
        flat = _normal(g, rows * (V + case["pad"]), dtype=dt, scale=2.0)
        s["logits"] = flat.as_strided((rows, V), (V + case["pad"], 1))
        tokens = torch.randint(0, V, (rows,), dtype=torch.int64, device=dev, generator=g)
        # the tokens are likely ones
        at = torch.arange(rows, device=dev)
        s["logits"][at, tokens] = (s["logits"][at, tokens].float() + _uniform(g, rows, hi=14.0)).to(dt)
        off = torch.randperm(rows, device=dev, generator=g)[:_skipped(case)]
        tokens[off] = -1
        s["tokens"] = tokens.to(torch.int32)
        if op == "logprobs_grad":
            # what a forward pass has left
            z = s["logits"].float() / case["temperature"]
            m = s["logits"].float().amax(-1)
            lp = z - (m / case["temperature"])[:, None]
            ls = torch.exp(lp).sum(-1).log()
            s["stats"] = torch.stack([m, ls], -1)
            lp -= ls[:, None]
            s["entropy"] = -(torch.exp(lp) * lp).sum(-1)
            s["dlogprobs"] = _normal(g, rows, dtype=torch.float32)
            s["dentropy"] = _normal(g, rows, dtype=torch.float32, scale=0.1) if case["entropy"] else None
            s["out"] = torch.empty(rows, V, dtype=dt, device=dev)
        return s
    d, rt = case["width"], TYPES[case["res"]]
    s["gain"] = 1.0 + _normal(g, d, dtype=torch.float32, scale=0.1)
    # a few columns of the residual stream are much larger than the others
    wide = (1.0 + 20.0 * (_uniform(g, d) < 0.01)).to(rt)
    s["rng"] = torch.tensor([int(seed) * 77777 + 5, int(seed) % 1000 + (3 << 33)], dtype=torch.int64, device=dev)
    if op == "norm":
        s["x"] = _normal(g, rows, d, dtype=dt)
        s["residual"] = _normal(g, rows, d, dtype=rt, scale=2.0) * wide
        s["out"] = [torch.empty(rows, d, dtype=rt, device=dev), torch.empty(rows, d, dtype=TYPES[case["y"]], device=dev)]
        if case["y"] == "e4m3":
            s["out"].append(torch.empty(rows, -(-d // case["group"]) if case["group"] else 1, device=dev))
    else:
        s["h"] = _normal(g, rows, d, dtype=rt, scale=2.0) * wide
        s["dy"], s["dh"] = _normal(g, rows, d, dtype=dt, scale=0.1), _normal(g, rows, d, dtype=rt, scale=0.1)
        s["out"] = torch.empty_like(s["h"]), torch.empty_like(s["dy"]), torch.empty_like(s["gain"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms

_LOW = 0xFFFFFFFF


def _philox_round(words, i):
    """One round of Philox4x32 (Salmon et al., 2011) on 32-bit words held in int64; products wrap at 64 bits."""
    c0, c1, c2, c3, k0, k1 = words
    a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
    c = ((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW
    return (*c, (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW)


def _keep(case, rng, rows, d):
    """Factor of every element: 0 where it is dropped."""
    threshold = int(round(case["drop"] * 65536))
    col = torch.arange(-(-d // 8), device=rng.device)[None, :].expand(rows, -1)
    row = torch.arange(rows, device=rng.device)[:, None].expand_as(col)
    fill = torch.zeros_like(col)
    seed, offset = rng[0], rng[1]
    words = (col, row, fill + (offset & _LOW), fill + ((offset >> 32) & _LOW), seed & _LOW, (seed >> 32) & _LOW)
    words = torch.stack(functools.reduce(_philox_round, range(10), words)[:4], -1)
    halves = torch.stack([words & 0xFFFF, words >> 16], -1).view(rows, -1)[:, :d]
    return (halves >= threshold) * (65536.0 / (65536 - threshold))


def _plain_norm(s):
    case = s["case"]
    x = s["x"].float()
    if case["drop"]:
        x = x * _keep(case, s["rng"], *x.shape)
    h = s["residual"].float() + x
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["gain"]
    h = h.to(s["residual"].dtype)
    if case["y"] != "e4m3":
        return [h, y.to(s["x"].dtype)]
    rows, d = y.shape
    n = case["group"] or d
    parts = torch.nn.functional.pad(y, (0, -d % n)).view(rows, -1, n)
    scales = parts.abs().amax(-1) / 448.0
    q = parts / torch.where(scales > 0, scales, torch.ones_like(scales))[..., None]
    return [h, q.view(rows, -1)[:, :d].to(torch.float8_e4m3fn), scales]


def _plain_norm_grad(s):
    case = s["case"]
    h, dy = s["h"].float(), s["dy"].float()
    rstd = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    n, t = h * rstd, dy * s["gain"]
    d = s["dh"].float() + rstd * (t - n * (t * n).mean(-1, keepdim=True))
    dx = d * _keep(case, s["rng"], *d.shape) if case["drop"] else d
    return [d.to(s["h"].dtype), dx.to(s["dy"].dtype), (dy * n).sum(0)]


def _plain_logprobs(s):
    case, logits = s["case"], s["logits"]
    T, V = case["temperature"], case["vocab"]
    z = logits.float()
    tok = s["tokens"].long()
    live = (tok >= 0) & (tok < V)
    m = z.amax(-1, keepdim=True)
    x = (z - m) / T
    e = torch.exp(x)
    S = e.sum(-1, keepdim=True)
    ls = torch.log(S)
    lp = x.gather(1, tok.clamp(0, V - 1)[:, None]) - ls
    zero = torch.zeros_like(lp)
    got = [torch.where(live[:, None], lp, zero)[:, 0], torch.where(live[:, None], torch.cat([m, ls], 1), zero)]
    if case["entropy"]:
        got.append(torch.where(live[:, None], ls - (e * x).sum(-1, keepdim=True) / S, zero)[:, 0])
    if case["top"]:
        # values and indices in one whole number: the largest value first, of equal ones the lowest index
        bits = (z + 0.0).view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        keys = (bits << 32) | (V - 1 - torch.arange(V, device=z.device))
        at = V - 1 - (keys.topk(case["top"], -1).values & _LOW)
        lp = x.gather(1, at) - ls
        got += [torch.where(live[:, None], at, -torch.ones_like(at)).to(torch.int32), torch.where(live[:, None], lp, torch.full_like(lp, float("-inf")))]
    return got


def _plain_logprobs_grad(s):
    case, logits = s["case"], s["logits"]
    T, V = case["temperature"], case["vocab"]
    tok = s["tokens"].long()
    live = (tok >= 0) & (tok < V)
    lp = (logits.float() - s["stats"][:, :1]) / T - s["stats"][:, 1:]
    p = torch.exp(lp)
    g = s["dlogprobs"][:, None]
    dz = -p * g
    if case["entropy"]:
        dz = dz - p * s["dentropy"][:, None] * (lp + s["entropy"][:, None])
    dz = torch.where(torch.arange(V, device=p.device)[None, :] == tok[:, None], dz + g, dz) / T
    return [torch.where(live[:, None], dz, torch.zeros_like(dz)).to(logits.dtype)]


def _plain_dpo(s):
    case = s["case"]
    B, k = case["B"], case["k"]
    starts = s["row_starts"].long()
    moved = torch.cumsum((s["pol"].double() - s["ref"].double()), 0)
    moved = torch.cat([moved.new_zeros(1), moved])
    sums = (moved[starts[1:]] - moved[starts[:-1]]).view(B, k)
    pos, neg = s["pos"].long(), s["neg"].long()
    x = BETA * (sums.gather(1, pos[:, None]) - sums.gather(1, neg[:, None]))[:, 0]
    loss = torch.clamp(-x, min=0) + torch.log1p(torch.exp(-x.abs()))
    step = BETA / B / (1.0 + torch.exp(x))
    which = torch.arange(k, device=x.device)[None, :]
    sign = (which == neg[:, None]).double() - (which == pos[:, None]).double()
    grad = torch.repeat_interleave((sign * step[:, None]).view(-1), starts[1:] - starts[:-1])
    return [loss.float(), grad.float()]


# ------------------------------------------------------------------------------------------------ one pass


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "logprobs": _plain_logprobs, "logprobs_grad": _plain_logprobs_grad,
                "dpo": _plain_dpo}[op](s)
    import paper_2410_18252_amd.rlgen as R
    if op == "norm":
        return list(R.rlgen_add_rms_norm(s["x"], s["gain"], EPS, residual=s["residual"], drop_p=case["drop"], rng=s["rng"], scale_group=case["group"],
                                         out=s["out"]))
    if op == "norm_grad":
        return list(R.rlgen_add_rms_norm_backward(s["h"], s["gain"], EPS, s["dy"], dh=s["dh"], drop_p=case["drop"], rng=s["rng"], out=s["out"]))
    if op == "logprobs":
        r = R.rlgen_token_logprobs(s["logits"], s["tokens"], case["temperature"], entropy=case["entropy"], n_top=case["top"])
        return [v for v in (r.logprobs, r.stats, r.entropy, r.top_tokens, r.top_logprobs) if v is not None]
    if op == "logprobs_grad":
        return [R.rlgen_token_logprobs_backward(s["logits"], s["tokens"], case["temperature"], s["stats"], s["dlogprobs"],
                                                entropy=s["entropy"] if case["entropy"] else None, dentropy=s["dentropy"], out=s["out"])]
    return list(R.rlgen_dpo_pairs(s["pol"], s["ref"], s["row_starts"], s["pos"], s["neg"], case["k"], BETA, weight=1.0 / case["B"], out=s["out"]))


# ------------------------------------------------------------------------------------------------ 64 bits


def _exact_factor(case, rng, rows, d):
    """The dropout factors, from numpy's unsigned arithmetic."""
    seed, offset = (int(v) & (2 ** 64 - 1) for v in rng.tolist())
    M, low = (np.uint64(0xD2511F53), np.uint64(0xCD9E8D57)), np.uint64(_LOW)
    words = np.zeros((4, rows, -(-d // 8)), np.uint64)
    words[0], words[1] = np.arange(words.shape[2], dtype=np.uint64)[None, :], np.arange(rows, dtype=np.uint64)[:, None]
    words[2], words[3] = np.uint64(offset & _LOW), np.uint64(offset >> 32)
    key = [seed & _LOW, seed >> 32]
    half = np.uint64(32)
    for _ in range(10):
        p, q = words[0] * M[0], words[2] * M[1]
        words = np.stack([(q >> half) ^ words[1] ^ np.uint64(key[0]), q & low, (p >> half) ^ words[3] ^ np.uint64(key[1]), p & low])
        key = [(key[0] + 0x9E3779B9) & _LOW, (key[1] + 0xBB67AE85) & _LOW]
    bits = np.ascontiguousarray(np.moveaxis(words, 0, -1).astype("<u4")).view("<u2").reshape(rows, -1)[:, :d]
    threshold = int(round(case["drop"] * 65536))
    return torch.from_numpy(np.where(bits >= threshold, 65536.0 / (65536 - threshold), 0.0))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "dpo":
        at, B, k = s["row_starts"].tolist(), case["B"], case["k"]
        pol, ref, pos, neg = (s[n].cpu().double().numpy() for n in ("pol", "ref", "pos", "neg"))
        loss, grad = np.zeros(B), np.zeros(at[-1])
        for b in range(B):
            i, j = b * k + int(pos[b]), b * k + int(neg[b])
            up, down = slice(at[i], at[i + 1]), slice(at[j], at[j + 1])
            x = BETA * (math.fsum(pol[up]) - math.fsum(ref[up]) - math.fsum(pol[down]) + math.fsum(ref[down]))
            loss[b] = math.log1p(math.exp(-x)) if x > -700 else -x
            t = BETA / B * (math.exp(-x) / (1.0 + math.exp(-x)) if x > -700 else 1.0)
            grad[up] -= t
            grad[down] += t
        return [torch.from_numpy(loss), torch.from_numpy(grad)]
    if op in ("logprobs", "logprobs_grad"):
        parts = [_exact_logits(case, s, a, min(case["rows"], a + 1024)) for a in range(0, case["rows"], 1024)]
        return [None if p[0] is None else torch.cat(p) for p in zip(*parts)]
    if case["drop"] and case["rows"] * case["width"] > 100e6:
        return None
    factor = _exact_factor(case, s["rng"], case["rows"], case["width"]).to(_device()) if case["drop"] else 1.0
    if op == "norm":
        h = s["residual"].double() + s["x"].double() * factor
        size = torch.sqrt(h.square().sum(-1, keepdim=True) / h.shape[1] + EPS)
        y = h / size * s["gain"].double()
        if case["y"] != "e4m3":
            return [h, y]
        n = case["group"] or h.shape[1]
        cuts = [y[:, a: a + n] for a in range(0, h.shape[1], n)]
        most = [c.abs().max(-1, keepdim=True).values / 448.0 for c in cuts]
        return [h, torch.cat([c / m for c, m in zip(cuts, most)], 1), torch.cat(most, 1)]
    h, dy, gain = s["h"].double(), s["dy"].double(), s["gain"].double()
    size = torch.sqrt(h.square().sum(-1, keepdim=True) / h.shape[1] + EPS)
    along = (dy * gain * h).sum(-1, keepdim=True) / h.shape[1] / size ** 3
    d = s["dh"].double() + dy * gain / size - h * along
    return [d, d * factor, (dy * h / size).sum(0)]


def _exact_logits(case, s, a, b):
    """Rows a..b, as a difference of log-sum-exps."""
    V, T = case["vocab"], case["temperature"]
    z = s["logits"][a:b].double()
    tok = s["tokens"][a:b].tolist()
    live = torch.tensor([0 <= t < V for t in tok], device=z.device)
    tok = torch.tensor([min(max(t, 0), V - 1) for t in tok], device=z.device)
    at = torch.arange(b - a, device=z.device)
    if case["op"] == "logprobs":
        z /= T
        lse = torch.logsumexp(z, -1)
        m = z.max(-1).values
        got = [torch.where(live, z[at, tok] - lse, 0.0), torch.where(live[:, None], torch.stack([m * T, lse - m], -1), 0.0)]
        if case["entropy"]:
            got.append(torch.where(live, lse - (torch.exp(z - lse[:, None]) * z).sum(-1), 0.0))
        if case["top"]:
            got += [None, torch.where(live[:, None], z.topk(case["top"], -1).values - lse[:, None], float("-inf"))]
        return got
    g = s["dlogprobs"][a:b].double()
    lp = z / T
    lp -= torch.logsumexp(lp, -1, keepdim=True)
    dz = torch.exp(lp)
    if case["entropy"]:
        H = -(dz * lp).sum(-1, keepdim=True)
        dz *= -(g[:, None] + s["dentropy"][a:b].double()[:, None] * (lp + H))
    else:
        dz *= -g[:, None]
    dz[at, tok] += g
    return [torch.where(live[:, None], dz / T, 0.0)]
