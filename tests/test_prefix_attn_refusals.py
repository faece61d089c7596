"""dcut_prefix_attn and dcut_enable_prefix_attn refuse bad arguments before they look at a device."""
import ctypes as C

import pytest

from paper_2607_14647_b200 import binding as b
from tests.test_rope_append_refusals import P, host_ctx


def call(h, groups=(1, P, P, P, 64), **kw):
    a = dict(q=P, k=P, v=P, num_pages=100, table=P, stride=64, ctx=P, cu=P, B=4, T_cap=9, scale=0.1, out=P, lse=None)
    a.update(kw)
    g = b.PrefixGroupsRec(*groups) if groups else None
    st = b._lib.dcut_prefix_attn(h, a["q"], a["k"], a["v"], a["num_pages"], a["table"], a["stride"], a["ctx"], a["cu"], a["B"], a["T_cap"],
                                 C.byref(g) if g is not None else None, a["scale"], a["out"], a["lse"], None)
    return st, b._lib.dcut_last_error(h).decode()


BAD = [(dict([(n, None)]), b.EINVAL) for n in ("q", "k", "v", "table", "ctx", "cu", "out", "groups")] + [
    (dict(groups=(0, P, P, P, 64)), b.EINVAL), (dict(groups=(5, P, P, P, 64)), b.EINVAL), (dict(groups=(1, None, P, P, 64)), b.EINVAL),
    (dict(groups=(1, P, None, P, 64)), b.EINVAL), (dict(groups=(1, P, P, None, 64)), b.EINVAL), (dict(groups=(1, P, P, P, 0)), b.ECAPACITY),
    (dict(groups=(1, P, P, P, 65)), b.ECAPACITY), (dict(B=0), b.EINVAL), (dict(B=9, T_cap=9), b.ECAPACITY), (dict(T_cap=3), b.EINVAL),
    (dict(T_cap=41), b.ECAPACITY), (dict(stride=0), b.ECAPACITY), (dict(stride=65), b.ECAPACITY), (dict(num_pages=0), b.EINVAL),
    (dict(num_pages=1 << 26), b.ECAPACITY), (dict(k=P + 64), b.EINVAL), (dict(v=P + 16), b.EINVAL), (dict(q=P + 8), b.EINVAL),
    (dict(out=P + 2), b.EINVAL), (dict(scale=0.0), b.EINVAL), (dict(scale=float("inf")), b.EINVAL), (dict(scale=float("nan")), b.EINVAL)]


@pytest.mark.parametrize("kw,status", BAD)
def test_refused(kw, status):
    h = host_ctx()
    st, msg = call(h, **kw)
    assert st == status and msg
    b._lib.dcut_destroy(h)


def test_enable_bounds():
    h = host_ctx()
    assert b._lib.dcut_enable_prefix_attn(None, 1) == b.EINVAL
    assert b._lib.dcut_enable_prefix_attn(h, 0) == b.EINVAL
    assert b._lib.dcut_enable_prefix_attn(h, 9) == b.ECAPACITY
    b._lib.dcut_destroy(h)
    h = host_ctx(n_q_heads=0, n_kv_heads=0, head_dim=0)
    assert b._lib.dcut_enable_prefix_attn(h, 1) == b.EINVAL and call(h)[0] == b.EINVAL
    b._lib.dcut_destroy(h)
