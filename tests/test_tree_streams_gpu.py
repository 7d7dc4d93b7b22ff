"""The calls of a round on a drafted tree on a stream that is not the current one, with the buffers that they make themselves."""
import numpy as np
import pytest
import torch

import tree_ref as R
from test_tree_attention_gpu import B, make  # noqa: F401

pytestmark = pytest.mark.gpu

LONG = 200_000_000  # cycles: a tenth of a second


def inputs(rng):
    d = R.verify_inputs(rng, 4, 9, 2000, torch.float32, T=0.8)
    adjust = {"bias_tokens": torch.tensor([[3], [4], [5], [6]], dtype=torch.int32, device="cuda"), "bias_values": torch.full((4, 1), 9.0, device="cuda"),
              "history": torch.from_numpy(rng.integers(0, 2000, (4, 500)).astype(np.int32)).cuda(), "prompt_len": torch.full((4,), 100, dtype=torch.int32, device="cuda"),
              "history_len": torch.full((4,), 500, dtype=torch.int32, device="cuda"), "frequency": torch.full((4,), 0.3, device="cuda")}
    return d, adjust


def test_default_outputs_belong_to_the_stream(B):  # noqa: F811
    """The current stream is busy: nothing that the calls do for their outputs may wait there and land on the results."""
    d = make(41, 3, 5, 4, 2, 64, 16, [100, 40, 333], torch.bfloat16)
    names = ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")
    v, adjust = inputs(np.random.default_rng(8))
    draft = {k: v[k] for k in ("draft_tokens", "parents")}
    ref = B.dssd_tree_attention(*[d[k] for k in names], parents=d["parents"], want_lse=True)
    ref2 = B.dssd_adjust_logits(v["target_logits"], **draft, **adjust)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    torch.cuda._sleep(LONG)
    got = B.dssd_tree_attention(*[d[k] for k in names], parents=d["parents"], want_lse=True, stream=s)
    got2 = B.dssd_adjust_logits(v["target_logits"], **draft, **adjust, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], ref[k]) for k in ref) and all(torch.equal(got2[k], ref2[k]) for k in ref2)


def test_scratch_belongs_to_the_stream(B):  # noqa: F811
    """The stream is busy when the calls are made: what they took for scratch is not given to the current stream meanwhile."""
    d = make(42, 3, 5, 4, 2, 64, 16, [100, 40, 333], torch.bfloat16)
    names = ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")
    v, adjust = inputs(np.random.default_rng(9))
    draft = {k: v[k] for k in ("draft_tokens", "parents")}
    ref = B.dssd_tree_attention(*[d[k] for k in names], parents=d["parents"], want_lse=True)
    ref2 = B.dssd_adjust_logits(v["target_logits"], **draft, **adjust)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(LONG)
    got = B.dssd_tree_attention(*[d[k] for k in names], parents=d["parents"], want_lse=True, stream=s)
    got2 = B.dssd_adjust_logits(v["target_logits"], **draft, **adjust, stream=s)
    sizes = [B.dssd_tree_attention_workspace_bytes(3, 5, 4, 2, 64), B.dssd_adjust_logits_workspace_bytes(4, 9, 2000, 500, 1)]
    other = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], ref[k]) for k in ref) and all(torch.equal(got2[k], ref2[k]) for k in ref2)
    assert all((x == 255).all() for x in other)
