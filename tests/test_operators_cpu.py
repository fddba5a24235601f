"""Host-only checks of the operators over pages and packed rows: what the entry points refuse before they touch the device, their
workspaces, and the plan's plain form on hand-made cases.  Never run beside a GPU: the pointers are no memory."""
import ctypes as C

import pytest
import torch

import window_reference as W

R = pytest.importorskip("paper_2410_18252_amd.rlgen", reason="librlgen.so not built")
D = C.c_void_p(256)          # aligned, never followed: every call below is refused
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-only checks")


def refuse(name, args, good, code, **kw):
    a = dict(good, **kw)
    assert getattr(R.lib, name)(*[a[k] for k in args]) == code, kw


PLAN = "ctx_lens new_lens S page_size free_pages n_free free_head page_table table_stride max_rows total_lens row_starts slots positions counts stream".split()
PLAN_GOOD = dict.fromkeys(PLAN, D) | dict(S=3, page_size=16, n_free=4, table_stride=2, max_rows=5, free_head=None, stream=None)


def test_plan_refuses():
    for name in ("ctx_lens", "new_lens", "free_pages", "page_table", "total_lens", "row_starts", "slots", "positions", "counts"):
        refuse("rlgen_plan_pages", PLAN, PLAN_GOOD, R.ERR_NULL, **{name: None})
    for kw in (dict(S=0), dict(S=-1), dict(page_size=0), dict(page_size=4), dict(page_size=24), dict(page_size=2048), dict(n_free=-1),
               dict(table_stride=0), dict(max_rows=-1)):
        refuse("rlgen_plan_pages", PLAN, PLAN_GOOD, R.ERR_BAD_ARG, **kw)


def test_rope_table_refuses():
    assert R.lib.rlgen_rope_table(None, 10, 8, 1e4, None) == R.ERR_NULL
    for args in ((0, 8, 1e4), (10, 7, 1e4), (10, 0, 1e4), (10, 258, 1e4), (10, 8, 0.0), (10, 8, float("nan")), (1 << 30, 8, 1e4)):
        assert R.lib.rlgen_rope_table(D, *args, None) == R.ERR_BAD_ARG, args


NORM = "qkv qkv_stride src rows hq hkv h q_gain k_gain eps rope max_pos r positions dtype".split()
NORM_GOOD = dict(qkv=D, qkv_stride=512, src=1, rows=4, hq=4, hkv=2, h=64, q_gain=D, k_gain=D, eps=1e-5, rope=D, max_pos=9, r=32, positions=D, dtype=1)
NORM_BAD = [dict(qkv_stride=504), dict(qkv_stride=516), dict(src=3), dict(src=-1), dict(dtype=0), dict(dtype=3), dict(rows=-1), dict(hq=0), dict(hq=3),
            dict(hkv=0), dict(h=24), dict(h=0), dict(h=272), dict(eps=-1.0), dict(eps=float("inf")), dict(r=7), dict(r=66), dict(r=-2), dict(max_pos=0),
            dict(qkv=C.c_void_p(264)), dict(rows=1 << 30)]


def test_norm_rope_refuses():
    args = NORM + "q qs k ks v vs pages n_pages page_size slots stream".split()
    good = NORM_GOOD | dict(q=D, qs=256, k=D, ks=128, v=D, vs=128, pages=D, n_pages=7, page_size=16, slots=D, stream=None)
    for kw in (dict(qkv=None), dict(q_gain=None), dict(k_gain=None), dict(rope=None), dict(positions=None), dict(q=None), dict(pages=None, k=None), dict(slots=None)):
        refuse("rlgen_qk_norm_rope", args, good, R.ERR_NULL, **kw)
    for kw in NORM_BAD + [dict(qs=248), dict(qs=260), dict(ks=120), dict(vs=132), dict(q=C.c_void_p(260)), dict(pages=C.c_void_p(264)), dict(n_pages=0),
                          dict(page_size=12), dict(page_size=2048), dict(n_pages=1 << 28)]:
        refuse("rlgen_qk_norm_rope", args, good, R.ERR_BAD_ARG, **kw)


def test_norm_rope_backward_refuses():
    args = NORM + "dq dqs dk dks dv dvs dqkv ds dqg dkg ws bytes stream".split()
    need = R.lib.rlgen_qk_norm_rope_backward_workspace(4, 64)
    assert need == 4 * 2 * 64 * 4 and R.lib.rlgen_qk_norm_rope_backward_workspace(-1, 64) == 0 and R.lib.rlgen_qk_norm_rope_backward_workspace(4, 300) == 0
    assert R.lib.rlgen_qk_norm_rope_backward_workspace(10 ** 6, 64) == R.lib.rlgen_qk_norm_rope_backward_workspace(10 ** 7, 64)
    good = NORM_GOOD | dict(dq=D, dqs=256, dk=D, dks=128, dv=D, dvs=128, dqkv=D, ds=512, dqg=D, dkg=D, ws=D, bytes=need, stream=None)
    for name in ("dq", "dk", "dv", "dqkv", "dqg", "dkg", "ws"):
        refuse("rlgen_qk_norm_rope_backward", args, good, R.ERR_NULL, **{name: None})
    for kw in NORM_BAD + [dict(dqs=252), dict(dks=8), dict(dvs=131), dict(ds=500), dict(ds=514), dict(dqkv=C.c_void_p(258))]:
        refuse("rlgen_qk_norm_rope_backward", args, good, R.ERR_BAD_ARG, **kw)
    refuse("rlgen_qk_norm_rope_backward", args, good, R.ERR_WORKSPACE, bytes=need - 1)
    refuse("rlgen_qk_norm_rope_backward", args, good, R.ERR_WORKSPACE, ws=C.c_void_p(264))


SHAPE_BAD = [dict(dtype=0), dict(dtype=3), dict(rows=-1), dict(hq=3), dict(hkv=0), dict(h=40), dict(h=512), dict(S=0), dict(longest=0), dict(window=-1),
             dict(sinks=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=C.c_void_p(264)), dict(qs=255), dict(qs=248), dict(longest=1 << 30),
             dict(S=1 << 28)]
SHAPE = "dtype rows hq hkv h starts S longest window sinks scale".split()
SHAPE_GOOD = dict(dtype=1, rows=9, hq=4, hkv=2, h=64, starts=D, S=2, longest=9, window=0, sinks=0, scale=0.1)


def test_window_attention_refuses():
    args = "q qs k ks v vs".split() + SHAPE + "out os lse stream".split()
    good = SHAPE_GOOD | dict(q=D, qs=256, k=D, ks=128, v=D, vs=128, out=D, os=256, lse=None, stream=None)
    for name in ("q", "k", "v", "starts", "out"):
        refuse("rlgen_window_attention", args, good, R.ERR_NULL, **{name: None})
    for kw in SHAPE_BAD + [dict(ks=120), dict(vs=129), dict(os=260), dict(out=C.c_void_p(257))]:
        refuse("rlgen_window_attention", args, good, R.ERR_BAD_ARG, **kw)


def test_window_attention_backward_refuses():
    args = "q qs k ks v vs out os lse do dos".split() + SHAPE + "dq dqs dk dks dv dvs ws bytes stream".split()
    need = R.lib.rlgen_window_attention_backward_workspace(9, 4, 2, 64, 2, 9, 0, 0)
    assert need >= 9 * 4 * 4
    long = R.lib.rlgen_window_attention_backward_workspace
    assert long(9000, 4, 2, 64, 1, 9000, 100, 4) > long(9000, 4, 2, 64, 1, 9000, 100, 0)       # the sinks' parts
    assert long(9000, 4, 2, 64, 1, 9000, 100, 10 ** 6) < 400 << 20                             # which stay bounded
    assert long(9, 4, 3, 64, 2, 9, 0, 0) == 0
    good = SHAPE_GOOD | dict(q=D, qs=256, k=D, ks=128, v=D, vs=128, out=D, os=256, lse=D, do=D, dos=256, dq=D, dqs=256, dk=D, dks=128, dv=D, dvs=128,
                             ws=D, bytes=need, stream=None)
    for name in ("q", "k", "v", "out", "lse", "do", "starts", "dq", "dk", "dv", "ws"):
        refuse("rlgen_window_attention_backward", args, good, R.ERR_NULL, **{name: None})
    for kw in SHAPE_BAD + [dict(dos=255), dict(dqs=8), dict(dks=136 - 1), dict(dvs=64), dict(do=C.c_void_p(264))]:
        refuse("rlgen_window_attention_backward", args, good, R.ERR_BAD_ARG, **kw)
    refuse("rlgen_window_attention_backward", args, good, R.ERR_WORKSPACE, bytes=need - 1)
    refuse("rlgen_window_attention_backward", args, good, R.ERR_WORKSPACE, ws=C.c_void_p(260))


def test_window_attention_paged_refuses():
    args = "q qs dtype rows hq hkv h pages n_pages page_size table stride starts totals S longest total window sinks scale out os lse ws bytes stream".split()
    size = R.lib.rlgen_window_attention_paged_workspace
    need = size(4, 2, 64, 2, 1, 4096, 0, 0)
    assert need > 0 and size(4, 2, 64, 2, 7, 4096, 0, 0) == 0 and size(4, 2, 64, 2, 1, 4096, 32, 0) == 0 and size(32, 32, 64, 512, 1, 4096, 0, 0) == 0
    assert size(4, 2, 60, 2, 1, 4096, 0, 0) == 0
    good = SHAPE_GOOD | dict(q=D, qs=256, pages=D, n_pages=9, page_size=16, table=D, stride=300, totals=D, longest=1, total=4096, out=D, os=256, lse=None,
                             ws=D, bytes=need, stream=None)
    for name in ("q", "pages", "table", "starts", "totals", "out"):
        refuse("rlgen_window_attention_paged", args, good, R.ERR_NULL, **{name: None})
    for kw in SHAPE_BAD + [dict(pages=C.c_void_p(264)), dict(n_pages=0), dict(page_size=7), dict(page_size=4), dict(page_size=2048), dict(stride=0),
                           dict(total=0), dict(n_pages=1 << 28)]:
        refuse("rlgen_window_attention_paged", args, good, R.ERR_BAD_ARG, **kw)
    for kw in (dict(ws=None), dict(bytes=need - 1), dict(ws=C.c_void_p(264))):
        refuse("rlgen_window_attention_paged", args, good, R.ERR_WORKSPACE, **kw)


def test_the_plans_plain_form():
    table = [[5, -7], [-7, -7], [2, -7]]
    total, starts, slots, pos, counts = W.plan([3, 0, 8], [6, 2, 1], 8, [9, 4, 1, 6], 0, table, 10)
    assert total == [9, 2, 9] and starts == [0, 6, 8, 9]
    assert slots == [43, 44, 45, 46, 47, 72, 32, 33, 8, -1] and pos == [3, 4, 5, 6, 7, 8, 0, 1, 8, 0]
    assert table == [[5, 9], [4, -7], [2, 1]] and counts == [9, 3, 9, 0]
