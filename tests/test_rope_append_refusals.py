"""dcut_rope_append refuses bad arguments before it looks at a device (so these run without a GPU)."""
import ctypes as C

import pytest

from paper_2607_14647_b200 import binding as b


def host_ctx(**kw):
    """A context record for argument checks: without a GPU dcut_create fails after the limits are stored, and the record
    is still returned (its message can be read); every refusal below comes before the device is touched."""
    lim = dict(max_B=8, max_gamma=4, n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=16, max_pages_per_req=64, vocab=0,
               hidden=0, intermediate=0)
    lim.update(kw)
    h, rec = C.c_void_p(None), b.Limits(*[lim[n] for n, _ in b.Limits._fields_])
    b._lib.dcut_create(C.byref(h), C.byref(rec), 0)
    assert h
    return h


P = 1 << 20          # an address that is aligned for everything and never read


def call(h, qkv=None, rope=None, groups=None, **kw):
    a = dict(q_out=P, k_cache=P, v_cache=P, num_pages=100, block_table=P, stride=64, cu_q=None, B=4, tok_req=P, tok_pos=P, T_cap=9)
    a.update(kw)
    x = dict(q=P, k=P, v=P, q_token_stride=1024, q_head_stride=128, k_token_stride=256, k_head_stride=128, v_token_stride=256, v_head_stride=128)
    x.update(qkv or {})
    r = dict(inv_freq=P, rotary_dim=128, interleaved=0, q_gain=None, k_gain=None, rms_eps=1e-6)
    r.update(rope or {})
    g = b.PrefixGroupsRec(*groups) if groups else None
    st = b._lib.dcut_rope_append(h, C.byref(b.Qkv(*[x[n] for n, _ in b.Qkv._fields_])), C.byref(b.Rope(*[r[n] for n, _ in b.Rope._fields_])),
                                 a["q_out"], a["k_cache"], a["v_cache"], a["num_pages"], a["block_table"], a["stride"],
                                 C.byref(g) if g is not None else None, a["cu_q"], a["B"], a["tok_req"], a["tok_pos"], a["T_cap"], None)
    return st, b._lib.dcut_last_error(h).decode()


BAD = [
    (dict(qkv=dict(k=None)), b.EINVAL), (dict(qkv=dict(q=None)), b.EINVAL), (dict(q_out=None), b.EINVAL),
    (dict(k_cache=None), b.EINVAL), (dict(block_table=None), b.EINVAL), (dict(tok_req=None), b.EINVAL), (dict(tok_pos=None), b.EINVAL),
    (dict(B=0), b.EINVAL), (dict(B=9), b.ECAPACITY), (dict(T_cap=0), b.EINVAL), (dict(num_pages=0), b.EINVAL),
    (dict(stride=0), b.ECAPACITY), (dict(stride=65), b.ECAPACITY),
    (dict(rope=dict(rotary_dim=24)), b.EINVAL), (dict(rope=dict(rotary_dim=144)), b.EINVAL), (dict(rope=dict(rotary_dim=-16)), b.EINVAL),
    (dict(rope=dict(inv_freq=None)), b.EINVAL), (dict(rope=dict(inv_freq=P + 4)), b.EINVAL),
    (dict(rope=dict(q_gain=P, rms_eps=-1.0)), b.EINVAL), (dict(rope=dict(k_gain=P, rms_eps=float("nan"))), b.EINVAL),
    (dict(rope=dict(q_gain=P + 8)), b.EINVAL),
    (dict(qkv=dict(q_token_stride=1028)), b.EINVAL), (dict(qkv=dict(v_head_stride=-128)), b.EINVAL), (dict(qkv=dict(k=P + 8)), b.EINVAL),
    (dict(k_cache=P + 64), b.EINVAL),
    (dict(groups=(0, P, P, None, 0)), b.EINVAL), (dict(groups=(5, P, P, None, 0)), b.EINVAL), (dict(groups=(1, None, P, None, 0)), b.EINVAL),
    (dict(groups=(1, P, None, None, 0)), b.EINVAL),
]


@pytest.mark.parametrize("kw,status", BAD)
def test_refused(kw, status):
    h = host_ctx()
    st, msg = call(h, **kw)
    assert st == status and msg
    b._lib.dcut_destroy(h)


def test_null_context_and_context_without_heads():
    assert b._lib.dcut_rope_append(None, None, None, None, None, None, 1, None, 1, None, None, 1, None, None, 1, None) == b.EINVAL
    h = host_ctx(n_q_heads=0, n_kv_heads=0, head_dim=0)
    st, msg = call(h)
    assert st == b.EINVAL and "attention shapes" in msg
    b._lib.dcut_destroy(h)
