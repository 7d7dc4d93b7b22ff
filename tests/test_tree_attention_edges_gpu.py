"""dssd_tree_attention where its scores leave the finite numbers: the same answer whether a sequence is taken in one piece or in several."""
import numpy as np
import pytest
import torch

from test_tree_attention_gpu import B, call, make  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,Hq,Hkv", [(3, 8, 2), (40, 16, 2)])
@pytest.mark.parametrize("length", [100, 4000])
def test_a_score_of_infinity_reaches_the_output(B, N, Hq, Hkv, length):  # noqa: F811
    """A visible key whose score overflows, or is infinite, makes its rows NaN; the others keep their bits."""
    d = make(31, 2, N, Hq, Hkv, 64, 16, [length, length // 2], torch.bfloat16, chain=True)
    good = call(B, d, want_lse=True)
    for big in (float("inf"), 1e38):
        e = dict(d, k_cache=d["k_cache"].clone(), q=d["q"].abs() + 0.5)
        ref = call(B, e, want_lse=True)
        t = length - 30
        e["k_cache"][int(d["block_table"][0, t // 16]), t % 16, 1] = big
        if big < float("inf"):
            e["q"] = e["q"].clone()
            e["q"][0] *= 16.0
        out = {"o": torch.full_like(d["q"], 7.0), "lse": torch.full((2, N, Hq), 7.0, device="cuda"), "flags": torch.zeros(2, dtype=torch.int32, device="cuda")}
        got = call(B, e, out=out)
        per = Hq // Hkv
        assert torch.isnan(got["o"][0, :, per: 2 * per]).all() and torch.isnan(got["lse"][0, :, per: 2 * per]).all()
        assert torch.isfinite(got["o"][0, :, :per].float()).all()
        assert torch.equal(got["o"][1], ref["o"][1]) and torch.equal(got["lse"][1], ref["lse"][1])
    assert torch.isfinite(good["o"].float()).all()


@pytest.mark.parametrize("length", [100, 4000])
def test_no_score_above_minus_infinity(B, length):  # noqa: F811
    """Where every visible key's score is -inf the sum is empty: lse is -inf, and o has no value (NaN)."""
    d = make(33, 1, 2, 4, 1, 64, 16, [length], torch.bfloat16, chain=True)
    d["q"] = d["q"].abs() + 0.5
    d["k_cache"][:] = float("-inf")
    d["k_new"][:] = float("-inf")
    got = call(B, d, want_lse=True)
    assert (got["lse"] == float("-inf")).all() and torch.isnan(got["o"]).all()
