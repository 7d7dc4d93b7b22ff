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


@pytest.mark.parametrize("handle", [False, True])
def test_a_round_on_another_stream(B, handle):  # noqa: F811
    """A whole round on a busy stream, given as a torch stream or as its handle, while the current one allocates and writes."""
    from paper_2507_12000_b200.tree import verify_round_tree

    v, adjust = inputs(np.random.default_rng(10))
    gen = torch.Generator(device="cuda").manual_seed(10)
    new = [torch.randn(3, 4, 9, 2, 16, generator=gen, device="cuda").half() for _ in range(2)]

    def round_(logits, stream):
        cache = [torch.zeros(3, 9, 16, 2, 16, device="cuda").half() for _ in range(2)]
        c = {"k_new": new[0], "v_new": new[1], "k_cache": cache[0], "v_cache": cache[1],
             "block_table": torch.arange(8, dtype=torch.int32, device="cuda").reshape(4, 2), "ctx_len": torch.tensor([0, 5, 16, 20], dtype=torch.int32, device="cuda")}
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(LONG)
        r = verify_round_tree(logits, v["draft_q"], v["draft_tokens"], v["parents"], v["uniforms"], v["uniforms_rs"], 0.8, adjust=adjust, cache=c,
                              stream=stream.cuda_stream if handle and stream is not None else stream)
        other = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (16, 144, 512, 1 << 12, 1 << 14, 1 << 16) for _ in range(8)]
        torch.cuda.synchronize()
        assert all((x == 255).all() for x in other)
        return dict(r, logits=logits, k=cache[0], v=cache[1])

    one = round_(v["target_logits"].clone(), None)
    two = round_(v["target_logits"].clone(), torch.cuda.Stream())
    assert all(torch.equal(one[k], two[k]) for k in one)


def test_what_is_no_stream_is_refused_before_anything_is_written(B):  # noqa: F811
    from paper_2507_12000_b200.tree import verify_round_tree

    v, adjust = inputs(np.random.default_rng(11))
    before = v["target_logits"].clone()
    with pytest.raises((TypeError, ValueError)):
        verify_round_tree(v["target_logits"], v["draft_q"], v["draft_tokens"], v["parents"], v["uniforms"], v["uniforms_rs"], 0.8, adjust=adjust,
                          stream="side")
    torch.cuda.synchronize()
    assert torch.equal(v["target_logits"], before)


def test_calls_on_two_streams_at_once(B):  # noqa: F811
    """Attention, adjusted logits and the verdict on two streams, call by call in turns, with the buffers that they make themselves."""
    names = ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")
    work = [(make(50 + i, 4, 7, 16, 2, 128, 16, [900, 40, 0, 5000], torch.bfloat16), *inputs(np.random.default_rng(50 + i))) for i in range(2)]

    def calls(i, stream):
        d, v, adjust = work[i]
        draft = {k: v[k] for k in ("draft_tokens", "parents")}
        yield B.dssd_tree_attention(*[d[k] for k in names], parents=d["parents"], want_lse=True, stream=stream)
        yield B.dssd_adjust_logits(v["target_logits"], **draft, **adjust, stream=stream)
        for replacement in (True, False):
            yield B.dssd_tree_verify(v["target_logits"], v["draft_q"], v["draft_tokens"], v["parents"], v["uniforms"], v["uniforms_rs"], 0.8,
                                     replacement=replacement, stream=stream)

    ref = [list(calls(i, None)) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = list(zip(*[calls(i, streams[i]) for i in range(2)]))
        torch.cuda.synchronize()
        for k, both in enumerate(got):
            for i in range(2):
                assert all(torch.equal(both[i][x], ref[i][k][x]) for x in ref[i][k])
