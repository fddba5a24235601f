"""The learner's operators past the last-level cache (rows of more than 256e6 bytes in all are streamed) and the norm's gradient at the widths whose threads
hold two and four pieces of a row, with more rows than blocks.  All rows are held against 64-bit forms, with the bounds of the smaller calls' tests, and bit by bit against the
same rows in calls below that size."""
import pytest
import torch

import test_gpu_add_norm as N

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF, F16 = torch.float32, torch.bfloat16, torch.float16
CACHE = 256e6


def normal(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def logits(seed, rows, V, dtype, pad=0, shift=0):
    """Rows `pad` elements apart from element `shift` of a buffer on, with likely tokens in them and a fifth of the rows left out."""
    flat = torch.full((shift + rows * (V + pad) + 16,), 99.0, dtype=dtype, device="cuda")
    z = flat.as_strided((rows, V), (V + pad, 1), shift)
    z.copy_(normal(seed, rows, V, dtype=dtype, scale=2.0))
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    tok = torch.randint(0, V, (rows,), generator=g, device="cuda")
    at = torch.arange(rows, device="cuda")
    z[at, tok] = (z[at, tok].float() + 12 * torch.rand(rows, generator=g, device="cuda")).to(dtype)
    tok[2::5] = -1
    return z, tok


def exact(z, T):
    """(log-probs, entropy, largest, log sum) in 64 bits."""
    x = z.double() / T
    ls = torch.logsumexp(x, -1, keepdim=True)
    lp = x - ls
    m = z.double().amax(-1, keepdim=True)
    return lp, -(lp.exp() * lp).sum(-1), m[:, 0], (ls - m / T)[:, 0]


SIZES = [(BF, 1100), (F16, 1100), (F32, 550)]
V = 128257


@pytest.mark.parametrize("n", [0, 5])
@pytest.mark.parametrize("dtype, rows", SIZES)
def test_logprobs(dtype, rows, n):
    T = 0.7
    z, tok = logits(rows + n, rows, V, dtype, pad=2, shift=3)
    assert rows * V * dtype.itemsize > CACHE
    got = R.rlgen_token_logprobs(z, tok.int(), T, n_top=n)
    live = tok >= 0
    step = 110                                                   # (over 64 rows of this length are taken whole, whatever their number)
    for a in range(0, rows, step):
        part = R.rlgen_token_logprobs(z[a:a + step], tok[a:a + step].int(), T, n_top=n)
        for name, p, q in zip(got._fields, got, part):
            assert p is None or torch.equal(p[a:a + step], q), name
        on = live[a:a + step]
        lp, H, m, ls = exact(z[a:a + step], T)
        mean = (lp.exp() * (lp + ls[:, None]).abs()).sum(-1)
        e = (V / 256 + 64) * U * (1 + 4 * mean)
        s = slice(a, a + step)
        assert torch.equal(got.stats[s, 0][on], m.float()[on])
        assert bool(((got.stats[s, 1] - ls).abs() <= e + 4 * U * ls.abs())[on].all())
        assert bool(((got.entropy[s] - H).abs() <= 4 * e + 4 * U * ls.abs())[on].all())
        want = lp.gather(1, tok[s].clamp(min=0)[:, None])[:, 0]
        assert bool(((got.logprobs[s] - want).abs() <= e + 8 * U * (want.abs() + ls.abs()))[on].all())
        if n:
            values, order = z[s].float().sort(dim=-1, descending=True, stable=True)
            assert torch.equal(got.top_tokens[s].long()[on], order[:, :n][on])
            want = lp.gather(1, order[:, :n])
            assert bool(((got.top_logprobs[s] - want).abs() <= (e + 4 * U * ls.abs())[:, None] + 4 * U * want.abs())[on].all())
    for t in (got.logprobs, got.entropy, got.stats):
        assert (t[~live] == 0).all()


@pytest.mark.parametrize("with_entropy", [False, True])
@pytest.mark.parametrize("dtype, rows", SIZES)
def test_logprobs_backward(dtype, rows, with_entropy):
    """Into an output that starts elsewhere within 16 bytes than the logits, and in place."""
    T, step = 0.8, 110
    z, tok = logits(rows, rows, V, dtype, pad=1, shift=5)
    assert 2 * rows * V * dtype.itemsize > CACHE > 2 * step * V * dtype.itemsize
    g, ge = normal(3, rows), normal(4, rows, scale=0.1) if with_entropy else None
    r = R.rlgen_token_logprobs(z, tok.int(), T)
    stats, H32 = r.stats, r.entropy
    flat = torch.full((1 + rows * (V + 2) + 16,), 99.0, dtype=dtype, device="cuda")
    out = flat.as_strided((rows, V), (V + 2, 1), 1)

    def call(s, to):
        return R.rlgen_token_logprobs_backward(z[s], tok[s].int(), T, stats[s], g[s], H32[s] if with_entropy else None, ge[s] if with_entropy else None, out=to)

    call(slice(0, rows), out)
    assert (flat[1:1 + rows * (V + 2)].view(rows, V + 2)[:, V:] == 99).all() and flat[0] == 99 and (flat[1 + rows * (V + 2):] == 99).all()
    eps, tiny = torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    for a in range(0, rows, step):
        s = slice(a, a + step)
        assert torch.equal(call(s, torch.empty(len(tok[s]), V, dtype=dtype, device="cuda")), out[s])
        lp, H, _, ls = exact(z[s], T)
        p, on = lp.exp(), tok[s] >= 0
        gs = g[s].double()[:, None]
        want, size = -p * gs, gs.abs().expand_as(p)
        if with_entropy:
            ges = ge[s].double()[:, None]
            want -= ges * p * (lp + H[:, None])
            size = size + ges.abs() * (lp.abs() + H[:, None])
        # p's exponent is off by its own roundings and by what the forward pass may be off in the log of the sum, the entropy by four times the latter
        mean = (p * (lp + ls[:, None]).abs()).sum(-1, keepdim=True)
        e = (V / 256 + 64) * U * (1 + 4 * mean)
        bound = p * size / T * (U * (16 + 8 * ((lp + ls[:, None]).abs() + ls.abs()[:, None])) + e)
        if with_entropy:
            bound += p * ges.abs() / T * 5 * e
        at = torch.arange(len(p), device="cuda"), tok[s].clamp(min=0)
        want[at] += gs[:, 0]
        bound[at] += 8 * U * gs[:, 0].abs() / T
        want = torch.where(on[:, None], want / T, 0.0)
        off = (out[s].double() - want).abs()
        assert bool((off <= eps * (1 + 100 * U) * want.abs() + bound + tiny).all())
        assert (out[s][~on] == 0).all()
    assert call(slice(0, rows), z) is z and torch.equal(z, out)


# bytes that a call moves: h, dh and dresidual, dy and dx
def rows_past_the_cache(width, dt, res):
    return int(CACHE / (width * (2 * dt.itemsize + 3 * res.itemsize))) + 77


@pytest.mark.parametrize("width, dt, res", [(4096, BF, BF), (4096, F16, F32), (2560, F32, F32), (520, BF, F32), (5120, BF, BF), (5120, BF, F32), (8192, F16, F16),
                                            (8192, F32, F32), (8200, F16, F32), (16384, BF, BF), (16384, BF, F32), (16384, F32, F32)])
def test_norm_backward(width, dt, res):
    """Every element of all gradients; in place; row gradients of the first rows alone, below the size."""
    rows, drop, eps = rows_past_the_cache(width, dt, res), 0.1, 1e-5
    h, gain = normal(1, rows, width, dtype=res), 1 + 0.2 * normal(2, width)
    dy, dh = normal(3, rows, width, dtype=dt, scale=0.3), normal(4, rows, width, dtype=res, scale=0.3)
    rng = torch.tensor([5, 6 << 40], dtype=torch.int64, device="cuda")
    few = rows // 3
    small = R.rlgen_add_rms_norm_backward(h[:few], gain, eps, dy[:few], dh[:few], drop, rng, out=(torch.empty_like(h[:few]), torch.empty_like(dy[:few]), torch.empty_like(gain)))
    got = R.rlgen_add_rms_norm_backward(h, gain, eps, dy, dh, drop, rng, out=(torch.empty_like(h), torch.empty_like(dy), torch.empty_like(gain)))
    assert torch.equal(got[0][:few], small[0]) and torch.equal(got[1][:few], small[1])
    # the mask as the forward pass draws it
    factor, _ = R.rlgen_add_rms_norm(torch.ones(rows, width, device="cuda"), None, 0.0, drop_p=drop, rng=rng)
    t = 65536 - round(65536 * drop)
    sums = [torch.zeros(width, dtype=torch.float64, device="cuda") for _ in range(2)]
    for a in range(0, rows, 1000):
        s = slice(a, a + 1000)
        h64, dh64, t64 = h[s].double(), dh[s].double(), dy[s].double() * gain.double()
        m = (factor[s] > 0) * (65536.0 / t)
        inv = 1 / torch.sqrt((h64 * h64).mean(-1, keepdim=True) + eps)
        d = dh64 + inv * (t64 - h64 * inv ** 2 * (t64 * h64).mean(-1, keepdim=True))
        parts = dh64.abs() + inv * t64.abs() + inv ** 3 * h64.abs() * (t64 * h64).abs().mean(-1, keepdim=True)
        for one, want, f, ty in ((got[0][s], d, 1.0, res), (got[1][s], d * m, m, dt)):
            e, tiny = N.half(ty)
            off = (one.double() - want).abs()
            assert bool((off <= e * (1 + 160 * U) * want.abs() + 160 * U * parts * f + tiny).all())
        sums[0] += (dy[s].double() * h64 * inv).sum(0)
        sums[1] += (dy[s].double() * h64 * inv).abs().sum(0)
    assert bool(((got[2] - sums[0]).abs() <= (40 + 60 + rows / 256 + 64) * U * sums[1]).all())
    dgain = torch.empty_like(gain)
    R.rlgen_add_rms_norm_backward(h, gain, eps, dy, dh, drop, rng, out=(dh, dy, dgain))
    assert torch.equal(dh, got[0]) and torch.equal(dy, got[1]) and torch.equal(dgain, got[2])


@pytest.mark.parametrize("dt, res", N.TYPES)
@pytest.mark.parametrize("width", [4104, 5120, 8192])
def test_norm_backward_with_two_pieces_to_a_thread(dt, res, width):
    for rows, drop, with_dh, pad in ((1, 0.0, True, 0), (3, 0.3, True, 8), (7, 0.1, False, 0)):
        N.check_backward(rows, width, dt, res, drop, with_dh, pad, seed=width + rows)


@pytest.mark.parametrize("dt, res", N.TYPES)
@pytest.mark.parametrize("width", [5120, 8200, 16384])
def test_norm_backward_with_more_rows_than_blocks(dt, res, width):
    N.check_backward(300, width, dt, res, 0.2, pad=16, seed=width)
    N.check_backward(517, width, dt, res, 0.0, with_dh=False, seed=width + 1)


def test_without_a_norm_past_the_cache():
    rows, width = 9000, 4096
    dh, rng = normal(1, rows, width, dtype=F32), torch.tensor([1, 2], dtype=torch.int64, device="cuda")
    factor, _ = R.rlgen_add_rms_norm(torch.ones(rows, width, device="cuda"), None, 0.0, drop_p=0.5, rng=rng)
    d, dx, none = R.rlgen_add_rms_norm_backward(None, None, 0.0, None, dh=dh, drop_p=0.5, rng=rng, dtype=BF)
    assert none is None and torch.equal(d, dh) and torch.equal(dx, (dh * factor).to(BF))
