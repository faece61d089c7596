"""dcut_lora in a context that found no tensor-map encoder (a record that never saw a driver is one)."""
import pytest
import torch

from paper_2607_14647_b200 import binding as b
from tests.test_lora_refusals import call
from tests.test_rope_append_refusals import host_ctx


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a GPU the record is a context that works, and the call's addresses are not real")
def test_it_is_refused_ahead_of_the_device():
    for kw in ({}, dict(n_q_heads=0, n_kv_heads=0, head_dim=0)):
        h = host_ctx(**kw)
        st, msg = call(h)
        assert st == b.ECUDA and "cuTensorMapEncodeTiled" in msg
        b._lib.dcut_destroy(h)
