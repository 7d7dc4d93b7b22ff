"""dssd_adjust_logits against the definition in float64.  Tolerance: five float32 operations on values of at most `mag`
and one rounding to the type of the logits, half a step each."""
import numpy as np
import pytest
import torch

import tree_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2507_12000_b200 import binding

    return binding


def inputs(rng, nb, N, V, dtype, L=50, K=7, masks=5, parents=True, penalties=True, holes=0.0):
    i32 = lambda *s, lo=0, hi=None: torch.from_numpy(rng.integers(lo, hi if hi is not None else V, s).astype(np.int32)).cuda()  # noqa: E731
    f = lambda *s: torch.from_numpy(rng.random(s).astype(np.float32)).cuda()  # noqa: E731
    d = {"logits": torch.from_numpy(rng.normal(0, 4, (nb, N, V))).to(dtype).cuda(), "draft_tokens": i32(nb, N - 1, hi=min(V, 6)),
         "parents": torch.from_numpy(R.random_parents(rng, nb, N, holes=holes)).cuda() if parents else None}
    if L:
        d["history"] = torch.from_numpy(np.minimum((V ** rng.random((nb, L))).astype(np.int32), V) - 1).cuda()
        d["history_len"], d["prompt_len"] = i32(nb, hi=L + 1), i32(nb, hi=L + 1)
    if penalties:
        d["repetition"], d["presence"], d["frequency"] = 1 + f(nb), f(nb) - 0.3, f(nb) - 0.2
    if K:
        d["bias_tokens"], d["bias_values"] = i32(nb, K, lo=-1), 10 * f(nb, K) - 5
    if masks:
        d["mask"] = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (masks, (V + 31) // 32)).astype(np.int32)).cuda()
        d["mask_row"] = i32(nb, N, lo=-1, hi=masks)
    return d


def call(B, d, **kw):
    names = ("draft_tokens", "parents", "repetition", "presence", "frequency", "bias_tokens", "bias_values", "mask", "mask_row")
    r = B.dssd_adjust_logits(d["logits"], d.get("history"), d.get("prompt_len"), d.get("history_len"), **{k: d.get(k) for k in names}, **kw)
    torch.cuda.synchronize()
    return r


def check(got, d, ref, mag, live, before, what=""):
    g = R.f64(got)
    eps = R.EPS[got.dtype]
    keep = ~np.broadcast_to(live[:, :, None], g.shape)
    assert ((g == before) | (np.isnan(g) & np.isnan(before)))[keep].all(), what + " rows without a node"
    with np.errstate(all="ignore"):
        # beyond the type's range a finite value is infinite
        lim = float(torch.finfo(got.dtype).max)
        r = np.where(np.abs(ref) > lim * (1 + eps), np.sign(ref) * np.inf, ref)
        tol = eps * np.abs(ref) + 5 * 2.0 ** -24 * mag
        ok = (g == r) | (np.isnan(g) & np.isnan(r)) | (np.abs(g - r) <= tol)
        edge = (np.abs(ref) + tol >= lim) & (np.sign(g) == np.sign(ref)) & (np.abs(g) >= lim * (1 - 2 * eps))
    bad = ~(ok | edge) & ~keep
    assert not bad.any(), (what, np.argwhere(bad)[:5], g[bad][:5], ref[bad][:5])


@pytest.mark.parametrize("nb,N,V,dtype,L,K,masks,parents", [
    (1, 1, 1, torch.float32, 1, 0, 0, False), (2, 3, 2, torch.bfloat16, 3, 1, 2, True), (3, 9, 31, torch.float32, 40, 5, 3, True),
    (2, 128, 33, torch.bfloat16, 9, 40, 4, True), (4, 5, 1000, torch.bfloat16, 300, 7, 0, False), (3, 7, 1025, torch.float32, 77, 0, 5, True),
    (2, 6, 4095, torch.bfloat16, 2100, 300, 6, True), (1, 9, 50272, torch.float32, 600, 32, 2, False), (5, 3, 9001, torch.bfloat16, 5000, 9, 1, True),
    (1, 2, 151936, torch.bfloat16, 100, 3, 1, True), (300, 2, 515, torch.float32, 5, 2, 3, True), (160, 3, 4104, torch.bfloat16, 20, 4, 9, True),
    (2, 3, 40000, torch.float32, 13000, 9, 2, True), (3, 2, 17000, torch.bfloat16, 20000, 2000, 0, False),
    (3, 4, 777, torch.float32, 0, 0, 4, True), (2, 3, 2048, torch.bfloat16, 0, 5, 0, False),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_against_the_definition(B, nb, N, V, dtype, L, K, masks, parents, in_place):
    rng = np.random.default_rng(nb * 7919 + N * 31 + V + L)
    d = inputs(rng, nb, N, V, dtype, L, K, masks, parents)
    ref, mag, live, bads = R.adjust(d)
    before = R.f64(d["logits"]) if in_place else np.full(d["logits"].shape, 3.0)
    out = {"logits": d["logits"] if in_place else torch.full_like(d["logits"], 3.0), "flags": torch.full((nb,), 99, dtype=torch.int32, device="cuda")}
    r = call(B, d, out=out)
    check(r["logits"], d, ref, mag, live, before)
    assert (r["flags"].cpu().numpy() == np.where(bads, B.ADJUST_FLAG_BAD_PARENT, 0)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("in_at,out_at", [(0, 0), (3, 3), (1, 2), (8, 0)])
def test_views(B, dtype, in_at, out_at):
    """Rows off every boundary, rows of another spacing, and what lies between rows left alone."""
    rng = np.random.default_rng(in_at * 10 + out_at)
    nb, N, V = 3, 5, 2051
    d = inputs(rng, nb, N, V, dtype)
    ref, mag, live, _ = R.adjust(d)
    a = torch.zeros(nb, N, V + 21, dtype=dtype, device="cuda")
    a[:, :, in_at:in_at + V] = d["logits"]
    o = torch.full((nb, N, V + 13), 7.0, dtype=dtype, device="cuda")
    call(B, dict(d, logits=a[:, :, in_at:in_at + V]), out={"logits": o[:, :, out_at:out_at + V]})
    check(o[:, :, out_at:out_at + V], d, ref, mag, live, np.full(ref.shape, 7.0))
    assert (o[:, :, :out_at] == 7).all() and (o[:, :, out_at + V:] == 7).all()
    whole = a.clone()
    v = whole[:, :, in_at:in_at + V]
    call(B, dict(d, logits=v), out={"logits": v})
    check(v, d, ref, mag, live, R.f64(d["logits"]))
    assert (whole[:, :, :in_at] == 0).all() and (whole[:, :, in_at + V:] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_odd_values(B, dtype):
    """Infinities, NaN and the type's lowest value, masked and not; untouched entries keep their bits."""
    rng = np.random.default_rng(1)
    d = inputs(rng, 4, 4, 640, dtype, L=200)
    x = d["logits"]
    x[:, :, ::7] = float("nan")
    x[:, :, 1::7] = float("-inf")
    x[:, :, 2::7] = torch.finfo(dtype).min
    x[:, :, 3::7] = float("inf")
    d["mask"][1] = 0  # nothing is allowed
    ref, mag, live, _ = R.adjust(d)
    r = call(B, d, out={"logits": torch.full_like(x, 3.0)})
    check(r["logits"], d, ref, mag, live, np.full(ref.shape, 3.0))


def test_flags_and_what_is_taken_instead(B):
    rng = np.random.default_rng(2)
    d = inputs(rng, 8, 4, 100, torch.float32, L=10)
    d["history"][0, 0], d["history_len"][0] = 100, 10
    d["draft_tokens"][1, 0], d["parents"][1] = -1, torch.tensor([0, 1, 2], dtype=torch.int32)
    d["bias_tokens"][2, 0] = 100
    d["history_len"][3], d["history_len"][4] = -1, 11
    d["repetition"][5], d["repetition"][6] = 0.0, float("nan")
    d["parents"][7] = torch.tensor([0, 2, 2], dtype=torch.int32)  # node 2 names itself, node 3 hangs under it
    d["mask_row"][0, 0] = 5
    ref, mag, live, bads = R.adjust(d)
    r = call(B, d, out={"logits": torch.full_like(d["logits"], 3.0), "flags": torch.zeros(8, dtype=torch.int32, device="cuda")})
    check(r["logits"], d, ref, mag, live, np.full(ref.shape, 3.0))
    assert bads.tolist() == [False] * 7 + [True]
    assert r["flags"].tolist() == [1 | 16, 1, 1, 4, 4, 8, 8, 2]


def test_the_last_of_a_tokens_biases_holds(B):
    x = torch.zeros(1, 1, 50, device="cuda")
    tok = torch.tensor([[7, 9, 7, 7, 9]], dtype=torch.int32, device="cuda")
    val = torch.tensor([[1.0, 2.0, 3.0, 4.0, 5.0]], device="cuda")
    r = B.dssd_adjust_logits(x, bias_tokens=tok, bias_values=val)["logits"][0, 0]
    assert r[7] == 4 and r[9] == 5 and r.abs().sum() == 9
    K = 1500
    tok = torch.full((1, K), 7, dtype=torch.int32, device="cuda")
    val = torch.arange(K, dtype=torch.float32, device="cuda")[None]
    assert B.dssd_adjust_logits(x, bias_tokens=tok, bias_values=val)["logits"][0, 0, 7] == K - 1


def test_mask_per_row_stream_and_graph(B):
    rng = np.random.default_rng(4)
    d = inputs(rng, 3, 4, 130, torch.bfloat16, masks=12)
    d["mask_row"] = None
    ref, mag, live, _ = R.adjust(d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r = call(B, d, stream=s)
    check(r["logits"], d, ref, mag, live, np.zeros(ref.shape))
    out = {"logits": torch.zeros_like(d["logits"])}
    ws = torch.full((B.dssd_adjust_logits_workspace_bytes(3, 4, 130, 50, 7),), 255, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call_args = dict(d)
        B.dssd_adjust_logits(call_args["logits"], d["history"], d["prompt_len"], d["history_len"], draft_tokens=d["draft_tokens"], parents=d["parents"],
                             repetition=d["repetition"], presence=d["presence"], frequency=d["frequency"], bias_tokens=d["bias_tokens"],
                             bias_values=d["bias_values"], mask=d["mask"], out=out, workspace=ws)
    d["logits"].mul_(0.5)
    d["history_len"].zero_()
    g.replay()
    torch.cuda.synchronize()
    ref, mag, live, _ = R.adjust(d)
    check(out["logits"], d, ref, mag, live, np.zeros(ref.shape))
