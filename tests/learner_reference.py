"""Plain forms of the learner's operators in 64 bits (numpy and torch on the CPU), sharing no code with the library."""
import numpy as np
import torch


def philox(counter, key):
    """Philox4x32 with ten rounds (Salmon et al., 2011) in Python's own whole numbers."""
    c, k, low = list(counter), list(key), 2 ** 32 - 1
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & low, (a >> 32) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def keep_factors(rows, width, drop_p, seed, offset, only=None):
    """[rows, width] factors of the dropout: 0, or the inverse of the quantised probability to stay."""
    low = 2 ** 32 - 1
    t = int(np.floor(drop_p * 65536 + 0.5))
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    out = np.zeros((rows, width))
    c = np.zeros((4, rows, width // 8), np.uint64)
    c[0], c[1] = np.arange(width // 8, dtype=np.uint64), np.arange(rows, dtype=np.uint64)[:, None]
    c[2], c[3] = np.uint64(offset & low), np.uint64(offset >> 32)
    k, s, m = [seed & low, seed >> 32], np.uint64(32), np.uint64(low)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = np.stack([(b >> s) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> s) ^ c[3] ^ np.uint64(k[1]), a & m])
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    for e in range(8):
        bits = (c[e // 2] >> np.uint64(16 * (e % 2))) & np.uint64(0xFFFF)
        out[:, e::8] = np.where(bits >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)
    return torch.from_numpy(out)


def add_norm(x, residual, factor, gain, eps):
    """(h, y, 1 / sqrt(mean h^2 + eps))."""
    h = x.double() * factor + (0 if residual is None else residual.double())
    inv = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return h, None if gain is None else h * inv * gain.double(), inv


def add_norm_backward(h, gain, eps, dy, dh, factor):
    h, d = h.double(), 0 if dh is None else dh.double()
    dgain = None
    if gain is not None:
        inv = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
        t = dy.double() * gain.double()
        d = d + inv * (t - h * inv ** 2 * (t * h).mean(-1, keepdim=True))
        dgain = (dy.double() * h * inv).sum(0)
    return d, d * factor, dgain


def logprobs(logits, T):
    """(log-probs of all tokens, entropy, largest logit, log sum) of rows; a row of -inf alone gives -inf, 0, -inf, -inf."""
    z = logits.double()
    m = z.max(-1, keepdim=True).values
    x = (z - torch.where(torch.isinf(m), torch.zeros_like(m), m)) / T
    e = torch.exp(x)
    ls = torch.log(e.sum(-1, keepdim=True))
    lp = torch.where(torch.isinf(ls), torch.full_like(x, float("-inf")), x - ls)
    p = torch.exp(lp)
    H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
    return lp, H, m[:, 0], ls[:, 0]


def logprobs_backward(logits, tokens, T, g, g_entropy):
    lp, H, m, _ = logprobs(logits, T)
    p = torch.exp(lp)
    d = -p * g.double()[:, None]
    if g_entropy is not None:
        d = d - g_entropy.double()[:, None] * torch.where(p > 0, p * (lp + H[:, None]), torch.zeros_like(p))
    V = logits.shape[1]
    live = ((tokens >= 0) & (tokens < V)) if tokens is not None else torch.ones(len(d), dtype=torch.bool)
    if tokens is not None:
        at = torch.arange(len(d))
        d[at, tokens.clamp(0, V - 1).long()] += g.double()
    return torch.where((live & (m > float("-inf")))[:, None], d / T, torch.zeros_like(d))


def top(logits, n):
    """The n largest of each row with the lowest index first among equal ones; NaN above everything."""
    z = torch.where(torch.isnan(logits), torch.full_like(logits.double(), float("inf")), logits.double()) + 0.0
    over = torch.isnan(logits).double()
    ids = []
    for a, b in zip(z.tolist(), over.tolist()):
        ids.append(sorted(range(len(a)), key=lambda i: (-b[i], -a[i], i))[:n])
    return torch.tensor(ids)


def dpo_pairs(pol, ref, starts, pos, neg, k, beta, weight):
    starts = [min(max(v, 0), len(pol)) for v in starts]
    loss, grad = torch.zeros(len(pos), dtype=torch.float64), torch.full((len(pol),), float("nan"), dtype=torch.float64)
    d = pol.double() - ref.double()
    for b in range(len(pos)):
        i, j = min(max(pos[b], 0), k - 1), min(max(neg[b], 0), k - 1)
        cut = [slice(starts[b * k + q], max(starts[b * k + q + 1], starts[b * k + q])) for q in range(k)]
        x = beta * (d[cut[i]].sum() - d[cut[j]].sum())
        loss[b] = torch.nn.functional.softplus(-x)
        for c in cut:
            grad[c] = 0
        step = weight * beta * torch.sigmoid(-x)
        grad[cut[i]] -= step
        grad[cut[j]] += step
    return loss, grad
