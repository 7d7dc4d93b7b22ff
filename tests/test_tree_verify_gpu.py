"""dssd_tree_verify against the definition in float64, against dssd_dsd_verify on chains, and against the law it has to keep."""
import numpy as np
import pytest
import torch

import tree_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2507_12000_b200 import binding

    return binding


def call(B, d, T, replacement, **kw):
    r = B.dssd_tree_verify(d["target_logits"], d["draft_q"], d["draft_tokens"], d["parents"], d["uniforms"], d["uniforms_rs"], T,
                           replacement=replacement, **kw)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy().astype(np.int64) for k, v in r.items()}


def same(got, ref):
    for k in ("accept_len", "path", "token", "edge_flags", "rs_flags"):
        assert (got[k] == ref[k]).all(), (k, np.argwhere(got[k] != ref[k])[:6], got[k], ref[k])


@pytest.mark.parametrize("nb,N,V,dtype,replacement", [
    (1, 1, 1, torch.float32, True), (3, 2, 2, torch.float32, False), (2, 5, 5, torch.bfloat16, True), (5, 17, 33, torch.float32, False),
    (1, 128, 129, torch.float32, True), (7, 33, 1000, torch.bfloat16, False), (40, 9, 4097, torch.float32, True), (170, 6, 1025, torch.bfloat16, True),
    (1, 16, 50272, torch.float32, True), (2, 64, 32000, torch.bfloat16, False), (330, 4, 515, torch.float32, False), (12, 24, 8191, torch.bfloat16, True),
    (1, 4, 300007, torch.bfloat16, True), (20, 7, 16411, torch.float32, False), (80, 3, 20001, torch.bfloat16, False),
])
def test_against_the_definition(B, nb, N, V, dtype, replacement):
    rng = np.random.default_rng(nb * 1000003 + N * 1009 + V)
    d = R.verify_inputs(rng, nb, N, V, dtype, T=0.8, sigma=0.9, replacement=replacement)
    same(call(B, d, 0.8, replacement), R.verify(d, 0.8, replacement))


@pytest.mark.parametrize("nb,N,V,dtype", [(9, 5, 4099, torch.bfloat16), (1, 9, 50272, torch.float32), (200, 3, 257, torch.float32)])
def test_a_chain_is_the_fused_round(B, nb, N, V, dtype):
    rng = np.random.default_rng(V)
    d = R.verify_inputs(rng, nb, N, V, dtype, T=0.7, parents=None)
    got = call(B, d, 0.7, True)
    ref = B.dssd_dsd_verify(d["target_logits"], d["draft_q"][:, : N - 1].contiguous(), d["draft_tokens"], d["uniforms"], d["uniforms_rs"], 0.7)
    torch.cuda.synchronize()
    for k in ("accept_len", "token", "edge_flags", "rs_flags"):
        assert (got[k] == ref[k].cpu().numpy()).all(), k
    chain = np.where(np.arange(N) <= got["accept_len"][:, None], np.arange(N), -1)
    assert (got["path"] == chain).all()
    listed = dict(d, parents=torch.arange(N - 1, dtype=torch.int32, device="cuda").expand(nb, N - 1).contiguous())
    same(call(B, listed, 0.7, True), got)


def test_a_chain_is_the_fused_round_on_rows_without_a_sum(B):
    rng = np.random.default_rng(17)
    d = R.verify_inputs(rng, 6, 3, 900, torch.float32, parents=None)
    x = d["target_logits"]
    x[0, 0, 5], x[1, 1, 7], x[2, 2], x[3, 0] = float("nan"), float("inf"), float("-inf"), float("-inf")
    d["draft_tokens"][4, 0] = 900
    d["uniforms"][:3] = 0.0
    got = call(B, d, 1.0, True)
    ref = B.dssd_dsd_verify(x, d["draft_q"][:, :2].contiguous(), d["draft_tokens"], d["uniforms"], d["uniforms_rs"], 1.0)
    torch.cuda.synchronize()
    for k in ("accept_len", "token", "rs_flags"):
        assert (got[k] == ref[k].cpu().numpy()).all(), k
    # (rows behind the walk's end are not looked at, so their flags may be missing here)
    assert ((got["edge_flags"] & ~ref["edge_flags"].cpu().numpy()) == 0).all()


@pytest.mark.parametrize("replacement", [True, False])
def test_the_first_token_follows_the_target(B, replacement):
    """Three candidates under the root: the emitted first token (accepted, or drawn after three rejections) has law p."""
    nb, V, T = 1 << 17, 5, 1.0
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.tensor([0.3, -1.0, 1.2, 0.0, -0.4], device="cuda")
    q = torch.tensor([0.5, 0.2, 0.05, 0.15, 0.1], device="cuda")
    if replacement:
        tok = torch.multinomial(q, nb * 3, replacement=True, generator=gen).reshape(nb, 3)
    else:
        tok = torch.multinomial(q.expand(nb, V), 3, replacement=False, generator=gen)
    d = {"target_logits": x.expand(nb, 4, V).contiguous(), "draft_q": q.expand(nb, 4, V).contiguous(), "draft_tokens": tok.int(),
         "parents": torch.zeros(nb, 3, dtype=torch.int32, device="cuda"), "uniforms": torch.rand(nb, 3, generator=gen, device="cuda"),
         "uniforms_rs": torch.rand(nb, generator=gen, device="cuda")}
    r = call(B, d, T, replacement)
    first = np.where(r["accept_len"] == 1, np.take_along_axis(tok.cpu().numpy(), np.maximum(r["path"][:, 1:2] - 1, 0), 1)[:, 0], r["token"])
    p = torch.softmax(x.double(), 0).cpu().numpy()
    freq = np.bincount(first, minlength=V) / nb
    assert (np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / nb)).all(), (freq, p)


def test_rows_out_of_order(B):
    """Rows that no finite log-sum-exp has, masks of the type's lowest value, bad tokens, bad parents, u = 1, q = 0 and NaN."""
    rng = np.random.default_rng(3)
    for dtype in (torch.float32, torch.bfloat16):
        d = R.verify_inputs(rng, 10, 6, 700, dtype, window=3, ragged=False)
        x, low = d["target_logits"], torch.finfo(dtype).min
        x[0, 0, 5] = float("nan")
        x[1, 0, 699] = float("inf")
        x[2, 0] = float("-inf")
        x[3, :, 1:] = low
        x[4, :, ::2] = float("-inf")
        d["draft_tokens"][5, 0] = -3
        d["draft_tokens"][6, 0] = 700
        d["parents"][7, 2] = 3      # itself
        d["parents"][8, 0] = -1     # and what hangs under it goes too
        d["uniforms"][9] = 1.0
        same(call(B, d, 1.0, True), R.verify(d, 1.0, True))
        d["draft_q"][9, 0, :] = 0
        d["draft_q"][8, 0, ::3] = float("nan")
        same(call(B, d, 1.0, False), R.verify(d, 1.0, False))


@pytest.mark.parametrize("T,shift", [(0.001, 0.0), (0.01, 3.0e4), (1.0, -3.0e4), (1e20, 0.0)])
def test_sums_beyond_the_range_of_float64(B, T, shift):
    """Scaled logits of thousands: the row is summed relative to its maximum.  At T = 1e20 only masked entries differ from the others."""
    rng = np.random.default_rng(12)
    d = R.verify_inputs(rng, 5, 4, 2000, torch.float32, window=2, ragged=False)
    d["target_logits"] += shift
    d["target_logits"][:, :, ::3] = float("-inf")
    same(call(B, d, T, True), R.verify(d, T, True))


def test_p_equal_to_q_falls_back(B):
    """A rejection by u = 1 where p = q leaves no mass: the token comes from p."""
    x = torch.zeros(2, 2, 64, device="cuda")
    q = torch.full((2, 2, 64), 1 / 64, device="cuda")
    d = {"target_logits": x, "draft_q": q, "draft_tokens": torch.zeros(2, 1, dtype=torch.int32, device="cuda"), "parents": None,
         "uniforms": torch.ones(2, 1, device="cuda"), "uniforms_rs": torch.tensor([0.0, 0.995], device="cuda")}
    r = call(B, d, 1.0, True)
    assert r["rs_flags"].tolist() == [2, 2] and r["token"].tolist() == [0, 63] and r["accept_len"].tolist() == [0, 0]


def test_every_sibling_refused_without_replacement(B):
    """Siblings that exhaust q: what is left of p is where q has no mass."""
    V = 8
    x = torch.zeros(1, 4, V, device="cuda")
    q = torch.zeros(1, 4, V, device="cuda")
    q[:, :, :3] = torch.tensor([0.5, 0.25, 0.25])
    d = {"target_logits": x, "draft_q": q, "draft_tokens": torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"),
         "parents": torch.zeros(1, 3, dtype=torch.int32, device="cuda"), "uniforms": torch.full((1, 3), 0.999, device="cuda"),
         "uniforms_rs": torch.tensor([0.3], device="cuda")}
    r = call(B, d, 1.0, False)
    same(r, R.verify(d, 1.0, False))
    assert r["accept_len"][0] in (0, 1)


def test_decisions_on_the_edge(B):
    """Uniforms put within float32's errors of a test's or a step's edge, from both sides: the verdict is the exact one."""
    rng = np.random.default_rng(31)
    nb, V, T = 400, 3001, 0.9
    d = R.verify_inputs(rng, nb, 2, V, torch.float32, T=T, sigma=1.2, parents=None)
    x = R.f64(d["target_logits"])[:, 0] / T
    p = np.exp(x - x.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    q = R.f64(d["draft_q"])[:, 0]
    tok = d["draft_tokens"][:, 0].cpu().numpy()
    ratio = p[np.arange(nb), tok] / q[np.arange(nb), tok]
    u = np.minimum(ratio, 0.9).astype(np.float32)
    u = np.where(np.arange(nb) % 2 == 0, np.nextafter(u, np.float32(0)), np.nextafter(u, np.float32(1)))
    rest = np.maximum(p - q, 0)
    cdf = np.cumsum(rest, axis=1)
    step = rng.integers(0, V, nb)
    ur = (cdf[np.arange(nb), step] / cdf[:, -1]).astype(np.float32)
    ur = np.clip(np.where(np.arange(nb) % 3 == 0, np.nextafter(ur, np.float32(0)), ur), 0, np.float32(1 - 2 ** -24))
    d["uniforms"] = torch.from_numpy(u[:, None].copy()).cuda()
    d["uniforms_rs"] = torch.from_numpy(ur).cuda()
    same(call(B, d, T, True), R.verify(d, T, True))


def test_strided_rows_other_stream_graph_and_garbage(B):
    rng = np.random.default_rng(8)
    d = R.verify_inputs(rng, 6, 7, 3001, torch.bfloat16)
    ref = R.verify(d, 0.9, True)
    wide = torch.full((6, 7, 3100), 9.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :, 11:3012] = d["target_logits"]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    same(call(B, dict(d, target_logits=wide[:, :, 11:3012]), 0.9, True, stream=s), ref)
    ws = torch.full((B.dssd_tree_verify_workspace_bytes(6, 7, 3001),), 255, dtype=torch.uint8, device="cuda")
    out = {k: torch.full((6,), 77, dtype=torch.int32, device="cuda") for k in ("accept_len", "token", "edge_flags", "rs_flags")}
    out["path"] = torch.full((6, 7), 77, dtype=torch.int32, device="cuda")
    same(call(B, d, 0.9, True, out=out, workspace=ws), ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.dssd_tree_verify(d["target_logits"], d["draft_q"], d["draft_tokens"], d["parents"], d["uniforms"], d["uniforms_rs"], 0.9, out=out, workspace=ws)
    d2 = R.verify_inputs(rng, 6, 7, 3001, torch.bfloat16)
    for k in d:
        d[k].copy_(d2[k])
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    same({k: v.cpu().numpy() for k, v in out.items()}, R.verify(d, 0.9, True))
