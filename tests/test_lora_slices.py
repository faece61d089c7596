"""An empty list of slices is refused like the other wrong ones."""
import pytest

from tests.test_operator_arguments import ctx  # noqa: F401  (a fixture)
from tests.test_operator_arguments_8bit import LORA, ctx8  # noqa: F401  (a fixture)


def test_no_slices(ctx8):  # noqa: F811
    with pytest.raises(AssertionError):
        ctx8.lora(**dict(LORA, slices=[]))
    assert not ctx8.calls
