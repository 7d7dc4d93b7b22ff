"""More of what the entry points of a round on a drafted tree refuse on the host (no GPU needed)."""
import pytest

from test_tree_boundary_cpu import B, P, append, verify  # noqa: F401


@pytest.mark.parametrize("T", [9e-31, 1e-38, 1e-45, 5e-324])
def test_the_verdict_refuses_temperatures_without_a_float32_inverse(B, T):  # noqa: F811
    """log2(e)/T of less than about 1e-38 is no float32, and a row's float32 pass would find no number in it."""
    assert verify(B, T=T) == B.DSSD_ERR_UNSUPPORTED
    assert verify(B, T=1e-30, workspace=None) == B.DSSD_ERR_WORKSPACE  # (checked after the temperature)


@pytest.mark.parametrize("kw", [
    dict(new_len=P + 4), dict(accept_len=2 * P), dict(accept_len=2 * P - 4), dict(path=2 * P - 28), dict(block_table=2 * P + 4), dict(flags=P),
    dict(ctx_len=2 * P + 4), dict(new_len=None, flags=P + 4), dict(flags=2 * P + 4),
])
def test_append_refuses_results_over_its_inputs(B, kw):  # noqa: F811
    """One CTA writes a sequence's results while others still look at its lengths, its path and its pages."""
    a = dict(ctx_len=P, accept_len=P + 64, path=P + 128, block_table=P + 1024, new_len=2 * P, flags=3 * P)
    a.update(kw)
    assert append(B, **a) == B.DSSD_ERR_INVALID_ARG
