"""dcut_linear8 refuses bad arguments before it looks at a device."""
import ctypes as C

import pytest

from paper_2607_14647_b200 import binding as b
from tests.test_rope_append_refusals import P, host_ctx

GOOD = dict(a=P, lda=112, a_scale=P, w=P, w2=None, ldw=112, w_scale=P, w2_scale=None, bias=None, bias2=None, residual=None, ldr=0, out=P, ldo=33, N=33,
            K=100, act=0)


def call(h, cu=P, B=4, T_cap=9, **kw):
    l = b.Linear8Args(*[dict(GOOD, **kw)[n] for n, _ in b.Linear8Args._fields_])
    st = b._lib.dcut_linear8(h, C.byref(l), cu, B, T_cap, None)
    return st, b._lib.dcut_last_error(h).decode()


BAD = [(dict([(n, None)]), b.EINVAL) for n in ("a", "w", "out", "cu", "a_scale", "w_scale")] + [
    (dict([(n, v)]), b.EINVAL) for n in ("B", "T_cap", "N", "K") for v in (0, -1)] + [(dict([(n, P + 8)]), b.EINVAL) for n in ("a", "w", "w2")] + [
    (dict([(n, P + 1)]), b.EINVAL) for n in ("out", "residual", "bias")] + [(dict([(n, P + 2)]), b.EINVAL) for n in ("a_scale", "w_scale")] + [
    (dict(bias2=P), b.EINVAL), (dict(w2=P), b.EINVAL), (dict(w2_scale=P), b.EINVAL), (dict(w2=P, w2_scale=P + 2), b.EINVAL),
    (dict(act=5), b.EINVAL), (dict(act=-1), b.EINVAL), (dict(lda=104), b.EINVAL), (dict(lda=96), b.EINVAL), (dict(ldw=104), b.EINVAL), (dict(ldw=0), b.EINVAL),
    (dict(lda=-112), b.EINVAL), (dict(lda=(1 << 32) + 16), b.EINVAL), (dict(ldo=32), b.EINVAL), (dict(residual=P, ldr=32), b.EINVAL),
    (dict(residual=P, ldr=34), b.EINVAL), (dict(N=(1 << 21) + 1, ldo=1 << 22), b.ECAPACITY), (dict(T_cap=(1 << 21) + 1), b.ECAPACITY)]


@pytest.mark.parametrize("kw,status", BAD)
def test_refused(kw, status):
    h = host_ctx()
    st, msg = call(h, **kw)
    assert st == status and msg
    b._lib.dcut_destroy(h)


def test_null_context_args_and_shapeless_context():
    assert b._lib.dcut_linear8(None, None, P, 1, 1, None) == b.EINVAL
    h = host_ctx()
    assert b._lib.dcut_linear8(h, None, P, 1, 1, None) == b.EINVAL
    b._lib.dcut_destroy(h)
    h = host_ctx(n_q_heads=0, n_kv_heads=0, head_dim=0)
    assert call(h)[0] == b.EINVAL
    b._lib.dcut_destroy(h)
