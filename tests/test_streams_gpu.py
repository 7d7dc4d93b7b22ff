"""The calls of a round on a stream that is not the current one, with the buffers that they make themselves."""
import pytest
import torch

import dssd_inputs as di
from gpu_util import to_device

pytestmark = pytest.mark.gpu

LONG = 200_000_000  # cycles: a tenth of a second


@pytest.fixture(scope="module")
def B():
    from paper_2507_12000_b200 import binding

    return binding


def calls(B, g, T, gamma, k):
    """Every call that makes outputs or scratch, on the same inputs; what each has left, by name."""
    row = torch.softmax(g["target_logits"][:, 0].float() / T, dim=-1).contiguous()
    n = (torch.arange(row.shape[0], device="cuda") % (gamma + 1)).int()
    torch.cuda.synchronize()

    def run(**kw):
        a = (g["target_logits"], g["draft_tokens"], g["draft_q_tok"], g["uniforms"])
        mass, _ = B.dssd_resample_shard_mass(row, g["draft_q"], n, gamma, **kw)
        return {"edge": B.dssd_edge_verify(*a, T, **kw), "topk": B.dssd_edge_verify_topk(*a, T, k, **kw),
                "bonus": B.dssd_edge_verify_bonus(*a, g["uniforms_rs"], T, **kw), "mass": {"mass": mass},
                "draw": B.dssd_device_resample(row, g["draft_q"], n, g["uniforms_rs"], gamma, **kw),
                "fused": B.dssd_dsd_verify(g["target_logits"], g["draft_q"], g["draft_tokens"], g["uniforms"], g["uniforms_rs"], T, **kw),
                "partial": B.dssd_edge_partial(g["target_logits"], g["draft_tokens"], 0, T, **kw)}
    return run


def same(got, ref):
    for c in ref:
        for k in ref[c]:
            assert (got[c][k] is None and ref[c][k] is None) or torch.equal(got[c][k], ref[c][k]), (c, k)


@pytest.fixture(scope="module")
def work(B):
    w = di.custom(B=40, gamma=3, V=20011, dtype="f32", temperature=0.9, sigma_d=0.9, seed=77)
    run = calls(B, to_device(di.generate(w)), w.temperature, w.gamma, 10)
    ref = run()
    torch.cuda.synchronize()
    return w, run, ref


def test_default_outputs_belong_to_the_stream(B, work):
    """The current stream is busy: the zeros that an output begins with may not wait there and land on the results."""
    w, run, ref = work
    s = torch.cuda.Stream()
    torch.cuda._sleep(LONG)
    got = run(stream=s)
    torch.cuda.synchronize()
    same(got, ref)


@pytest.mark.parametrize("handle", [False, True])
def test_scratch_belongs_to_the_stream(B, work, handle):
    """The stream is busy when the calls are made: what they took for scratch is not given to the current stream meanwhile."""
    w, run, ref = work
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(LONG)
    got = run(stream=s.cuda_stream if handle else s)
    sizes = [B.dssd_edge_verify_workspace_bytes(w.B, w.gamma, w.V), B.dssd_device_resample_workspace_bytes(w.B, w.gamma, w.V),
             B.dssd_dsd_verify_workspace_bytes(w.B, w.gamma, w.V), B.dssd_edge_partial_workspace_bytes(w.B, w.gamma, w.V), 1 << 16]
    other = [torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]
    torch.cuda.synchronize()
    same(got, ref)
    assert all((x == 255).all() for x in other)


@pytest.mark.parametrize("handle", [0, 1, 2])
def test_handles_of_the_default_streams(B, work, handle):
    """The legacy default stream by both of its handles, and the thread's own."""
    w, run, ref = work
    got = run(stream=handle)
    torch.cuda.synchronize()
    same(got, ref)
