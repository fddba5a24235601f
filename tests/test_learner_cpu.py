"""Host-only checks of the learner's operators: what the entry points refuse before they touch the device, and the plain forms on cases with known
answers.  Never run beside a GPU: the pointers are no memory."""
import ctypes as C

import pytest
import torch

import learner_reference as L

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
D = C.c_void_p(256)          # aligned, never followed: every call below is refused
host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="host-only checks")


def refuse(name, args, good, code, **kw):
    a = dict(good, **kw)
    assert getattr(R.lib, name)(*[a[k] for k in args]) == code, kw


NORM = "x xs dtype r rs res rows width drop rng gain eps h hs y ys ydt scales group stream".split()
NORM_GOOD = dict(x=D, xs=64, dtype=1, r=D, rs=64, res=1, rows=3, width=64, drop=0.1, rng=D, gain=D, eps=1e-5, h=D, hs=64, y=D, ys=64, ydt=1, scales=None, group=0,
                 stream=None)
SHAPE_BAD = [dict(dtype=3), dict(dtype=-1), dict(res=2), dict(res=3), dict(rows=-1), dict(rows=1 << 23), dict(width=0), dict(width=60), dict(width=16392),
             dict(drop=-0.1), dict(drop=1.1), dict(drop=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(rng=C.c_void_p(260)), dict(gain=C.c_void_p(264))]


@host_only
def test_add_rms_norm_refuses():
    name = "rlgen_add_rms_norm"
    for kw in (dict(x=None), dict(h=None, y=None), dict(rng=None), dict(gain=None), dict(ydt=3)):
        refuse(name, NORM, NORM_GOOD, R.ERR_NULL, **kw)
    for kw in SHAPE_BAD + [dict(xs=56), dict(xs=68), dict(rs=56), dict(hs=65), dict(ys=8), dict(x=C.c_void_p(264)), dict(y=C.c_void_p(258)),
                           dict(r=C.c_void_p(260)), dict(h=C.c_void_p(260)), dict(ydt=0), dict(ydt=2), dict(ydt=4), dict(xs=1 << 31),
                           dict(ydt=3, scales=D, group=16), dict(ydt=3, scales=D, group=256), dict(ydt=3, scales=D, group=-32),
                           dict(ydt=3, scales=C.c_void_p(258))]:
        refuse(name, NORM, NORM_GOOD, R.ERR_BAD_ARG, **kw)


@host_only
def test_add_rms_norm_backward_refuses():
    args = "h hs res dy dys dtype dh dhs rows width drop rng gain eps dr drs dx dxs dg ws bytes stream".split()
    size = R.lib.rlgen_add_rms_norm_backward_workspace
    need = size(100, 64)
    assert need >= 64 * 4 and size(3, 64) == 0 and size(-1, 64) == 0 and size(100, 60) == 0 and size(100, 20000) == 0
    assert size(10 ** 6, 4096) == size(8 * 10 ** 6, 4096) < 64 << 20
    good = dict(h=D, hs=64, res=1, dy=D, dys=64, dtype=1, dh=D, dhs=64, rows=100, width=64, drop=0.1, rng=D, gain=D, eps=1e-5, dr=D, drs=64, dx=D, dxs=64, dg=D,
                ws=D, bytes=need, stream=None)
    for kw in (dict(h=None), dict(dy=None), dict(dg=None), dict(rng=None), dict(dr=None, dx=None), dict(gain=None), dict(gain=None, dg=None),
               dict(gain=None, dg=None, dy=None, dh=None)):
        refuse("rlgen_add_rms_norm_backward", args, good, R.ERR_NULL, **kw)
    for kw in SHAPE_BAD + [dict(hs=56), dict(dys=65), dict(dhs=4), dict(drs=60), dict(dxs=60), dict(dx=C.c_void_p(264)), dict(dg=C.c_void_p(258))]:
        refuse("rlgen_add_rms_norm_backward", args, good, R.ERR_BAD_ARG, **kw)
    for kw in (dict(ws=None), dict(bytes=need - 1), dict(ws=C.c_void_p(264))):
        refuse("rlgen_add_rms_norm_backward", args, good, R.ERR_WORKSPACE, **kw)


LOGITS_BAD = [dict(rows=-1), dict(rows=1 << 24), dict(V=0), dict(V=(1 << 24) + 1, zs=1 << 25), dict(zs=99), dict(zs=1 << 31), dict(dtype=3), dict(dtype=-1),
              dict(z=C.c_void_p(257)), dict(dtype=0, z=C.c_void_p(258)), dict(T=0.0), dict(T=-1.0), dict(T=1e-7), dict(T=float("inf")), dict(T=float("nan"))]


@host_only
def test_token_logprobs_refuses():
    args = "z zs dtype rows V tokens T lp stats entropy n ids top ws bytes stream".split()
    good = dict(z=D, zs=100, dtype=1, rows=3, V=100, tokens=D, T=0.7, lp=D, stats=D, entropy=D, n=5, ids=D, top=D, ws=None, bytes=0, stream=None)
    size = R.lib.rlgen_token_logprobs_workspace
    need = size(1, 3, 100000, 5)
    assert need > 0 and size(1, 300, 100000, 5) == 0 and size(1, 3, 1000, 5) == 0 and size(3, 3, 100000, 5) == 0 and size(1, 3, 100000, 65) == 0
    for kw in (dict(ws=None, bytes=need), dict(ws=D, bytes=need - 1), dict(ws=C.c_void_p(264), bytes=need)):
        refuse("rlgen_token_logprobs", args, good, R.ERR_WORKSPACE, V=100000, zs=100000, **kw)
    for kw in (dict(z=None), dict(stats=None), dict(tokens=None), dict(lp=None), dict(ids=None), dict(top=None)):
        refuse("rlgen_token_logprobs", args, good, R.ERR_NULL, **kw)
    for kw in LOGITS_BAD + [dict(n=-1), dict(n=65), dict(n=11, V=10)]:
        refuse("rlgen_token_logprobs", args, good, R.ERR_BAD_ARG, **kw)


@host_only
def test_token_logprobs_backward_refuses():
    args = "z zs dtype rows V tokens T stats entropy g ge d ds stream".split()
    good = dict(z=D, zs=100, dtype=1, rows=3, V=100, tokens=D, T=0.7, stats=D, entropy=D, g=D, ge=D, d=D, ds=100, stream=None)
    for kw in (dict(z=None), dict(stats=None), dict(tokens=None), dict(entropy=None), dict(g=None, ge=None), dict(d=None)):
        refuse("rlgen_token_logprobs_backward", args, good, R.ERR_NULL, **kw)
    for kw in LOGITS_BAD + [dict(ds=99), dict(d=C.c_void_p(257)), dict(rows=1 << 21, V=8192 * 8, zs=1 << 17, ds=1 << 17)]:
        refuse("rlgen_token_logprobs_backward", args, good, R.ERR_BAD_ARG, **kw)


@host_only
def test_dpo_pairs_refuses():
    args = "pol ref rows starts B k pos neg beta weight loss grad stream".split()
    good = dict(pol=D, ref=D, rows=9, starts=D, B=2, k=2, pos=D, neg=D, beta=0.1, weight=1.0, loss=D, grad=D, stream=None)
    for name in ("pol", "ref", "starts", "pos", "neg", "loss", "grad"):
        refuse("rlgen_dpo_pairs", args, good, R.ERR_NULL, **{name: None})
    for kw in (dict(rows=-1), dict(B=0), dict(k=0), dict(B=1 << 22), dict(B=1 << 20, k=1 << 12), dict(beta=float("nan")), dict(weight=float("inf"))):
        refuse("rlgen_dpo_pairs", args, good, R.ERR_BAD_ARG, **kw)


def test_the_generators_published_answers():
    """Philox4x32 with ten rounds: the published known answers of counter and key 0, all ones, and the digits of pi."""
    assert L.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert L.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert L.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]
    f = L.keep_factors(3, 24, 0.5, 5 + (7 << 32), 9 + (11 << 32))
    w = L.philox([2, 1, 9, 11], [5, 7])
    assert f[1, 16:].tolist() == [2.0 if b >= 32768 else 0.0 for v in w for b in (v & 0xFFFF, v >> 16)]


def test_the_plain_forms_against_autograd():
    g = torch.Generator().manual_seed(1)

    def leaf(*shape):
        return torch.randn(*shape, generator=g, dtype=torch.float64).requires_grad_()

    x, r, gain = leaf(3, 16), leaf(3, 16), leaf(16)
    f = L.keep_factors(3, 16, 0.4, 1, 2)
    h, y, _ = L.add_norm(x, r, f, gain, 1e-5)
    dy, dh = torch.randn(3, 16, generator=g, dtype=torch.float64), torch.randn(3, 16, generator=g, dtype=torch.float64)
    want = torch.autograd.grad((y * dy).sum() + (h * dh).sum(), (r, x, gain))
    for a, b in zip(L.add_norm_backward(h.detach(), gain.detach(), 1e-5, dy, dh, f), want):
        assert torch.allclose(a, b, rtol=1e-10, atol=1e-12)
    z, tok = leaf(4, 9), torch.tensor([3, -1, 0, 8])
    gl, ge = torch.randn(4, generator=g, dtype=torch.float64), torch.randn(4, generator=g, dtype=torch.float64)
    lp = torch.log_softmax(z / 0.7, -1)
    live = tok >= 0
    total = (torch.where(live, gl * lp[torch.arange(4), tok.clamp(min=0)], 0) + torch.where(live, ge * -(lp.exp() * lp).sum(-1), 0)).sum()
    assert torch.allclose(L.logprobs_backward(z.detach(), tok, 0.7, gl, ge), torch.autograd.grad(total, z)[0], rtol=1e-10, atol=1e-12)
    pol = leaf(12)
    ref = torch.randn(12, generator=g, dtype=torch.float64)
    loss, grad = L.dpo_pairs(pol.detach(), ref, [0, 3, 7, 12], [2], [0], 3, 0.3, 1.5)
    d = pol - ref
    want = -torch.nn.functional.logsigmoid(0.3 * (d[7:].sum() - d[:3].sum()))
    assert torch.allclose(loss[0], want) and torch.allclose(grad, torch.autograd.grad(1.5 * want, pol)[0])
