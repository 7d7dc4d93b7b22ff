"""More of what the entry points of a round on a drafted tree refuse on the host (no GPU needed)."""
import pytest

from test_tree_boundary_cpu import B, verify  # noqa: F401


@pytest.mark.parametrize("T", [9e-31, 1e-38, 1e-45, 5e-324])
def test_the_verdict_refuses_temperatures_without_a_float32_inverse(B, T):  # noqa: F811
    """log2(e)/T of less than about 1e-38 is no float32, and a row's float32 pass would find no number in it."""
    assert verify(B, T=T) == B.DSSD_ERR_UNSUPPORTED
    assert verify(B, T=1e-30, workspace=None) == B.DSSD_ERR_WORKSPACE  # (checked after the temperature)
