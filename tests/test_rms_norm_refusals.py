"""dcut_rms_norm refuses bad arguments before it looks at a device."""
import ctypes as C

import pytest

from paper_2607_14647_b200 import binding as b
from tests.test_rope_append_refusals import P, host_ctx

GOOD = dict(x=P, ldx=104, residual=None, ldr=0, gain=P, gain_plus_one=0, normed=1, rms_eps=1e-6, width=100, h_out=None, ldh=0, out=P + 4096, ldo=100,
            out8=None, ld8=0, scale8=None)


def call(h, cu=P, B=4, T_cap=9, **kw):
    n = b.NormArgs(*[dict(GOOD, **kw)[f] for f, _ in b.NormArgs._fields_])
    st = b._lib.dcut_rms_norm(h, C.byref(n), cu, B, T_cap, None)
    return st, b._lib.dcut_last_error(h).decode()


BAD = [(dict(x=None), b.EINVAL), (dict(out=None), b.EINVAL), (dict(out8=P, ld8=112), b.EINVAL), (dict(scale8=P), b.EINVAL), (dict(normed=0), b.EINVAL),
       (dict(rms_eps=0.0), b.EINVAL), (dict(rms_eps=-1.0), b.EINVAL), (dict(rms_eps=float("nan")), b.EINVAL), (dict(rms_eps=float("inf")), b.EINVAL),
       (dict(ldx=99), b.EINVAL), (dict(ldx=-104), b.EINVAL), (dict(ldx=(1 << 32) + 8), b.EINVAL), (dict(ldo=99), b.EINVAL), (dict(residual=P, ldr=99), b.EINVAL),
       (dict(h_out=P + 8192, ldh=96), b.EINVAL), (dict(out8=P + 8192, ld8=96, scale8=P), b.EINVAL), (dict(x=P + 1), b.EINVAL), (dict(gain=P + 1), b.EINVAL),
       (dict(out=P + 4097), b.EINVAL), (dict(out8=P + 8193, ld8=112, scale8=P + 2), b.EINVAL), (dict(h_out=P, ldh=112), b.EINVAL),
       (dict(out=P, ldo=112), b.EINVAL), (dict(residual=P + 8192, ldr=104, h_out=P + 8192, ldh=112), b.EINVAL), (dict(h_out=P + 4096, ldh=100), b.EINVAL),
       (dict(residual=P + 4096, ldr=100), b.EINVAL), (dict(width=32769, ldx=40000, ldo=40000), b.ECAPACITY), (dict(T_cap=(1 << 30) + 1), b.ECAPACITY)] + [
    (dict([(n, v)]), b.EINVAL) for n in ("B", "T_cap", "width") for v in (0, -1)]


@pytest.mark.parametrize("kw,status", BAD)
def test_refused(kw, status):
    h = host_ctx()
    st, msg = call(h, **kw)
    assert st == status and msg
    b._lib.dcut_destroy(h)


def test_null_context_and_args():
    assert b._lib.dcut_rms_norm(None, None, P, 1, 1, None) == b.EINVAL
    h = host_ctx()
    assert b._lib.dcut_rms_norm(h, None, P, 1, 1, None) == b.EINVAL
    b._lib.dcut_destroy(h)
