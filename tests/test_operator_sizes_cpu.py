"""How large a call of the attention over packed rows and pages may be: what fits one launch is not refused.  Where there is no GPU a call that is
accepted ends at its launch.  Never run beside one: the pointers are no memory."""
import pytest
import torch

from test_operators_cpu import D, R, SHAPE, SHAPE_GOOD

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-only checks")


def call(name, **kw):
    hq, hkv, h = kw["hq"], kw["hkv"], kw["h"]
    a = SHAPE_GOOD | dict(q=D, k=D, v=D, out=D, lse=D, do=D, dq=D, dk=D, dv=D, pages=D, table=D, totals=D, n_pages=9, page_size=16, stride=8, total=128, stream=None,
                          qs=hq * h, ks=hkv * h, vs=hkv * h, os=hq * h, dos=hq * h, dqs=hq * h, dks=hkv * h, dvs=hkv * h, ws=D, bytes=1 << 60) | kw
    args = {"rlgen_window_attention": "q qs k ks v vs".split() + SHAPE + "out os lse stream".split(),
            "rlgen_window_attention_backward": "q qs k ks v vs out os lse do dos".split() + SHAPE + "dq dqs dk dks dv dvs ws bytes stream".split(),
            "rlgen_window_attention_paged": "q qs dtype rows hq hkv h pages n_pages page_size table stride starts totals S longest total window sinks scale out os "
                                            "lse ws bytes stream".split()}[name]
    return getattr(R.lib, name)(*[a[k] for k in args])


# (rows or new tokens of all sequences, sequences, longest, query heads, kv heads, dims)
PACKED = [(262144, 1, 262144, 64, 8, 128), (200000, 1, 200000, 24, 2, 64), (131072, 1, 131072, 16, 1, 128), (8192, 4096, 2, 32, 32, 64), (5000, 100, 1 << 24, 8, 8, 64),
          (2 ** 24 - 128, 1, 2 ** 24 - 128, 8, 8, 64), (9, 2 ** 21 - 8, 9, 8, 8, 64)]
DECODE = [(4096, 32, 32), (8192, 16, 16), (16384, 8, 8), (32768, 64, 8), (2 ** 23 - 1, 8, 8)]


@pytest.mark.parametrize("rows, S, longest, hq, hkv, h", PACKED)
def test_packed_rows_of_any_size_that_a_launch_holds(rows, S, longest, hq, hkv, h):
    kw = dict(rows=rows, S=S, longest=longest, hq=hq, hkv=hkv, h=h)
    assert call("rlgen_window_attention", **kw) == R.ERR_DEVICE
    assert call("rlgen_window_attention_backward", **kw) == R.ERR_DEVICE
    if longest <= rows:
        assert call("rlgen_window_attention_paged", **kw) == R.ERR_DEVICE


@pytest.mark.parametrize("S, hq, hkv", DECODE)
def test_single_tokens_of_any_number_that_a_launch_holds(S, hq, hkv):
    assert call("rlgen_window_attention_paged", rows=S, S=S, longest=1, hq=hq, hkv=hkv, h=64) == R.ERR_DEVICE


def test_what_no_launch_holds_is_refused():
    for kw in (dict(rows=9, S=2 ** 21, longest=9, hq=8, hkv=8), dict(rows=1 << 20, S=1 << 12, longest=1 << 20, hq=8, hkv=8), dict(rows=9, S=1 << 28, longest=9, hq=4, hkv=4)):
        for name in ("rlgen_window_attention", "rlgen_window_attention_backward", "rlgen_window_attention_paged"):
            assert call(name, h=64, **kw) == R.ERR_BAD_ARG, (name, kw)
    # two blocks to a tile of keys beyond 96 dims
    kw = dict(rows=9, S=2 ** 20, longest=9, hq=8, hkv=8)
    assert call("rlgen_window_attention_backward", h=96, **kw) == R.ERR_DEVICE and call("rlgen_window_attention_backward", h=112, **kw) == R.ERR_BAD_ARG
    assert call("rlgen_window_attention_paged", rows=9, S=2 ** 26 // 8, longest=1, hq=8, hkv=8, h=64) == R.ERR_BAD_ARG
