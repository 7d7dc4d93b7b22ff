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


def test_spacing_along_dimensions_of_one_entry(B):  # noqa: F811
    """Keys and values of one head, cut out of tensors of different shapes: the spacing along the one head does not matter."""
    d = make(35, 2, 3, 4, 1, 64, 16, [100, 33], torch.bfloat16)
    ref = call(B, d)["o"]
    both = torch.cat([d["k_new"], d["v_new"]], dim=2)
    e = dict(d, k_new=both[:, :, :1], v_new=both.transpose(1, 2).contiguous().transpose(1, 2)[:, :, 1:])
    if e["k_new"].stride()[:2] != e["v_new"].stride()[:2]:
        e["v_new"] = torch.as_strided(both, (2, 3, 1, 64), (both.stride(0), both.stride(1), 8, 1), 64)
    assert e["k_new"].stride() != e["v_new"].stride() and torch.equal(e["v_new"], d["v_new"])
    assert torch.equal(call(B, e)["o"], ref)
    cache = [torch.zeros(1, 40, 16, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.arange(20, dtype=torch.int32, device="cuda").reshape(2, 10)
    kn, vn = e["k_new"][None], e["v_new"][None]
    odd = torch.as_strided(cache[1], cache[1].shape, (8,) + cache[1].stride()[1:])
    B.dssd_cache_append(kn, vn, cache[0], odd, table, d["ctx_len"], torch.full((2,), 2, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for c, new in zip(cache, (d["k_new"], d["v_new"])):
        for b, n in enumerate((100, 33)):
            for i in range(3):
                assert torch.equal(c[0, int(table[b, (n + i) // 16]), (n + i) % 16], new[b, i])
