"""What the linear layers refuse, and what the refusal says (no GPU)."""
import pytest

from paper_2607_14647_b200 import binding as b
from tests import test_linear8_refusals as linear8
from tests import test_linear_refusals as linear
from tests.test_rope_append_refusals import host_ctx


@pytest.mark.parametrize("call", [linear.call, linear8.call])
def test_a_context_without_attention_shapes_is_told_what_it_lacks(call):
    h = host_ctx(n_q_heads=0, n_kv_heads=0, head_dim=0)
    st, msg = call(h)
    assert st == b.EINVAL and "without attention shapes" in msg and "encoder" not in msg
    b._lib.dcut_destroy(h)
