"""dcut_lora refuses bad arguments before it looks at a device."""
import ctypes as C

import pytest

from paper_2607_14647_b200 import binding as b
from tests.test_rope_append_refusals import P, host_ctx

GOOD = dict(x=P, ldx=104, a=P, lda=104, b=P, scale=None, adapter=P, n_adapters=3, rank=16, n_slices=2, slice_end=(20, 44), K=100, act=0, gated=0, base=P,
            ldbase=44, out=P + 4096, ldo=44)


def call(h, cu=P, B=4, T_cap=9, **kw):
    v = dict(GOOD, **kw)
    v["slice_end"] = (C.c_int * 4)(*v["slice_end"])
    l = b.LoraArgs(*[v[n] for n, _ in b.LoraArgs._fields_])
    st = b._lib.dcut_lora(h, C.byref(l), cu, B, T_cap, None)
    return st, b._lib.dcut_last_error(h).decode()


BAD = [(dict([(n, None)]), b.EINVAL) for n in ("x", "a", "b", "adapter", "base", "out", "cu")] + [
    (dict([(n, v)]), b.EINVAL) for n in ("B", "T_cap", "K", "n_adapters", "n_slices", "rank") for v in (0, -1)] + [
    (dict([(n, P + 8)]), b.EINVAL) for n in ("x", "a", "b")] + [(dict([(n, P + 1)]), b.EINVAL) for n in ("base", "out")] + [
    (dict([(n, P + 2)]), b.EINVAL) for n in ("scale", "adapter")] + [
    (dict(rank=4), b.EINVAL), (dict(rank=20), b.EINVAL), (dict(rank=136), b.ECAPACITY), (dict(n_slices=5), b.EINVAL),
    (dict(slice_end=(20, 20)), b.EINVAL), (dict(slice_end=(44, 20)), b.EINVAL), (dict(slice_end=(0, 44)), b.EINVAL), (dict(act=5), b.EINVAL), (dict(act=-1), b.EINVAL),
    (dict(gated=1), b.EINVAL), (dict(gated=1, n_slices=1, slice_end=(43,)), b.EINVAL), (dict(gated=1, n_slices=3, slice_end=(22, 44, 60), ldbase=60), b.EINVAL),
    (dict(ldx=100), b.EINVAL), (dict(ldx=96), b.EINVAL), (dict(lda=101), b.EINVAL), (dict(lda=-104), b.EINVAL), (dict(lda=(1 << 32) + 8), b.EINVAL),
    (dict(ldbase=43), b.EINVAL), (dict(ldo=43), b.EINVAL), (dict(out=P, ldo=48), b.EINVAL), (dict(out=P, gated=1, slice_end=(22, 44)), b.EINVAL),
    (dict(out=P, base=P + 4096), b.EINVAL), (dict(slice_end=(20, (1 << 21) + 1), ldbase=1 << 22, ldo=1 << 22), b.ECAPACITY), (dict(T_cap=(1 << 21) + 1), b.ECAPACITY),
    (dict(B=8193), b.ECAPACITY), (dict(n_adapters=(1 << 22) + 1), b.ECAPACITY), (dict(ldo=1 << 32), b.EINVAL), (dict(ldbase=1 << 32), b.EINVAL)]


@pytest.mark.parametrize("kw,status", BAD)
def test_refused(kw, status):
    h = host_ctx()
    st, msg = call(h, **kw)
    assert st == status and msg
    b._lib.dcut_destroy(h)


def test_null_context_and_args():
    assert b._lib.dcut_lora(None, None, P, 1, 1, None) == b.EINVAL
    h = host_ctx()
    assert b._lib.dcut_lora(h, None, P, 1, 1, None) == b.EINVAL
    b._lib.dcut_destroy(h)
