"""How far the sizes of the linear layers, the norm and the adapters go, and what a refusal says (no GPU: a size that is taken is shown by
an address that is refused later on)."""
import pytest

from paper_2607_14647_b200 import binding as b
from tests import test_linear8_refusals as linear8
from tests import test_linear_refusals as linear
from tests import test_lora_refusals as lora
from tests import test_rms_norm_refusals as norm
from tests.test_rope_append_refusals import P, host_ctx


@pytest.mark.parametrize("call", [linear.call, linear8.call])
def test_a_context_without_attention_shapes_is_told_what_it_lacks(call):
    h = host_ctx(n_q_heads=0, n_kv_heads=0, head_dim=0)
    st, msg = call(h)
    assert st == b.EINVAL and "without attention shapes" in msg and "encoder" not in msg
    b._lib.dcut_destroy(h)


FAR = 1 << 32
LIMITS = [(call, name, most, over, more) for call in (linear.call, linear8.call) for name, most, over, more in (
    ("N", 1 << 21, b.ECAPACITY, dict(ldo=FAR)), ("K", 1 << 30, b.ECAPACITY, dict(lda=FAR, ldw=FAR)), ("T_cap", 1 << 21, b.ECAPACITY, {}),
    ("lda", FAR, b.EINVAL, {}), ("ldw", FAR, b.EINVAL, {}))] + [
    (lora.call, name, most, over, more) for name, most, over, more in (
        ("K", 1 << 30, b.ECAPACITY, dict(ldx=FAR, lda=FAR)), ("T_cap", 1 << 21, b.ECAPACITY, {}), ("B", 8192, b.ECAPACITY, {}), ("n_adapters", 1 << 22, b.ECAPACITY, {}),
        ("ldx", FAR, b.EINVAL, {}), ("lda", FAR, b.EINVAL, {}), ("ldbase", FAR - 1, b.EINVAL, {}), ("ldo", FAR - 1, b.EINVAL, {}))] + [
    (norm.call, "width", 32768, b.ECAPACITY, dict(ldx=FAR, ldo=FAR)), (norm.call, "T_cap", 1 << 30, b.ECAPACITY, {}), (norm.call, "ldx", FAR, b.EINVAL, {})]


@pytest.mark.parametrize("call,name,most,over,more", LIMITS)
def test_sizes_go_as_far_as_stated(call, name, most, over, more):
    h = host_ctx()
    odd = dict(base=P + 1) if call is lora.call else dict(out=P + 4097)
    st, msg = call(h, **dict(more, **{name: most}, **odd))
    assert st == b.EINVAL and "2-byte aligned" in msg
    st, msg = call(h, **dict(more, **{name: most + 16}, **odd))
    assert st == over and "2-byte aligned" not in msg
    b._lib.dcut_destroy(h)


def test_columns_of_the_adapters():
    h = host_ctx()
    for N, status in ((1 << 21, b.EINVAL), ((1 << 21) + 1, b.ECAPACITY)):
        st, msg = lora.call(h, slice_end=(20, N), ldbase=1 << 22, ldo=1 << 22, base=P + 1)
        assert st == status and ("2-byte aligned" in msg) == (status == b.EINVAL)
    b._lib.dcut_destroy(h)
