"""dssd_tree_attention against the definition in float64.

Tolerance of o: the weights are rounded to the inputs' type (half a step, relative to sum w |v|), o is rounded once more, and a
score of D float32 products is off by at most D 2^-24 times the sum of their magnitudes, which moves weights and their sum by as much each;
2^-21 covers the exponentials and the sums' own roundings.  binary16 weights below 2^-14 lose up to 2^-25 each, relative to the largest weight."""
import numpy as np
import pytest
import torch

import tree_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2507_12000_b200 import binding

    return binding


def make(seed, nb, N, Hq, Hkv, D, page, lens, dtype, window=4, chain=False, holes=0.0, qscale=1.0):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    per = max(1, -(-max(lens) // page))
    total = nb * per + 2
    return {"q": qscale * t(nb, N, Hq, D), "k_new": t(nb, N, Hkv, D), "v_new": t(nb, N, Hkv, D), "k_cache": t(total, page, Hkv, D),
            "v_cache": t(total, page, Hkv, D), "ctx_len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
            "block_table": torch.from_numpy(rng.permutation(total)[: nb * per].reshape(nb, per).astype(np.int32)).cuda(),
            "parents": None if chain else torch.from_numpy(R.random_parents(rng, nb, N, window, holes=holes)).cuda()}


def call(B, d, scale=None, **kw):
    names = ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")
    r = B.dssd_tree_attention(*[d[k] for k in names], parents=d["parents"], scale=scale, **kw)
    torch.cuda.synchronize()
    return r


def check(got, d, scale=None, lse=None, keep=0.0):
    scale = d["q"].shape[3] ** -0.5 if scale is None else scale
    o, ls, live, wv, big = R.attention(d, scale)
    g = R.f64(got)
    eps, D, dt = R.EPS[got.dtype], got.shape[3], got.dtype
    n = int(d["ctx_len"].max()) + got.shape[1]
    off = 2.0 * D * 2.0 ** -24 * big[..., None] + 2.0 ** -21
    tol = (eps + 2 * off) * wv + eps * np.abs(o) * (1 + eps)
    if dt == torch.float16:
        tol = tol + (n * 2.0 ** -25 + 2.0 ** -25) * float(max(d["v_cache"].abs().max(), d["v_new"].abs().max()))
    bad = ~(np.abs(g - o) <= tol) & live[:, :, None, None]
    assert not bad.any(), (np.argwhere(bad)[:5], g[bad][:5], o[bad][:5], tol[bad][:5])
    assert (g[~live] == keep).all()
    if lse is not None:
        bad = ~(np.abs(R.f64(lse) - ls) <= off[..., 0] + 2.0 ** -22 * (1 + np.abs(ls))) & live[:, :, None]
        assert not bad.any(), (np.argwhere(bad)[:5], R.f64(lse)[bad][:5], ls[bad][:5])


SHAPES = [
    # nb, N, Hq, Hkv, D, page, lens
    (1, 1, 1, 1, 8, 1, [0]), (1, 1, 8, 1, 64, 16, [1]), (2, 1, 4, 4, 128, 16, [127, 128]), (3, 5, 6, 2, 64, 16, [0, 129, 300]),
    (2, 9, 14, 2, 96, 48, [511, 40]), (1, 64, 8, 1, 128, 32, [700]), (2, 128, 2, 2, 64, 128, [5, 257]), (1, 33, 32, 2, 128, 8, [1030]),
    (1, 128, 16, 1, 128, 64, [200]), (4, 3, 5, 1, 40, 7, [13, 255, 256, 64]), (1, 2, 128, 1, 128, 256, [900]), (2, 17, 8, 8, 120, 3, [90, 2]),
    (1, 4, 32, 8, 128, 16, [5000]), (40, 2, 4, 2, 64, 16, [3 * i for i in range(40)]), (1, 16, 3, 3, 16, 512, [1500]), (2, 12, 12, 1, 80, 24, [385, 1]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_definition(B, shape, dtype):
    nb, N, Hq, Hkv, D, page, lens = shape
    d = make(N * 100 + D, nb, N, Hq, Hkv, D, page, lens, dtype)
    r = call(B, d, want_lse=True)
    check(r["o"], d, lse=r["lse"])
    assert (r["flags"] == 0).all()


@pytest.mark.parametrize("N", [1, 5, 40])
def test_a_chain(B, N):
    d = make(N, 3, N, 8, 2, 128, 16, [0, 77, 640], torch.bfloat16, chain=True)
    r = call(B, d, want_lse=True)
    check(r["o"], d, lse=r["lse"])
    listed = dict(d, parents=torch.arange(N - 1, dtype=torch.int32, device="cuda").expand(3, N - 1).contiguous())
    assert torch.equal(call(B, listed)["o"], r["o"])


def test_large_scores_and_another_scale(B):
    """Scores of a few hundred: one key takes all the weight; and a maximum that keeps growing along the cache."""
    d = make(3, 2, 4, 4, 2, 64, 16, [300, 520], torch.bfloat16, qscale=8.0)
    check(call(B, d, scale=0.7)["o"], d, scale=0.7)
    ramp = torch.linspace(0.1, 4.0, d["k_cache"].shape[0], device="cuda")[:, None, None, None]
    d["k_cache"] = (d["k_cache"].abs() * ramp).bfloat16()
    d["q"] = d["q"].abs()
    order = torch.arange(d["block_table"].numel(), dtype=torch.int32, device="cuda").reshape(d["block_table"].shape)
    d["block_table"] = order
    check(call(B, d, scale=0.05)["o"], d, scale=0.05)


def test_garbage_in_unused_places(B):
    """NaN and infinity behind a sequence's end, in pages of nobody, in rows without a node; rows without a node keep what they held."""
    for lens, page in (([5, 130, 0], 16), ([200, 63, 17], 64)):
        d = make(5, 3, 9, 4, 2, 128, page, lens, torch.bfloat16, holes=0.2)
        ref = call(B, d)["o"]
        used = torch.zeros(d["k_cache"].shape[:2], dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            for t in range(n):
                used[int(d["block_table"][b, t // page]), t % page] = True
        for k in ("k_cache", "v_cache"):
            d[k][~used] = float("nan") if k == "v_cache" else float("inf")
        live = [[w is not None for w in R.ways(p, 9)[0]] for p in d["parents"].tolist()]
        dead = ~torch.tensor(live, device="cuda")
        for k in ("q", "k_new", "v_new"):
            d[k][dead] = float("nan")
        d["block_table"][:, max(-(-n // page) for n in lens):] = -5
        out = {"o": torch.full_like(d["q"], 2.5), "flags": torch.zeros(3, dtype=torch.int32, device="cuda")}
        call(B, d, out=out)
        assert torch.equal(out["o"][~dead], ref[~dead]) and (out["o"][dead] == 2.5).all() and (out["flags"] == 0).all()


def test_without_a_cache(B):
    """No pages at all, a table without columns, a table of pages that do not exist: the nodes see each other."""
    d = make(21, 3, 7, 4, 2, 64, 16, [0, 0, 0], torch.bfloat16)
    ref = call(B, d)["o"]
    check(ref, d)
    none = torch.empty(0, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    e = dict(d, k_cache=none, v_cache=none, block_table=torch.empty(3, 0, dtype=torch.int32, device="cuda"))
    assert torch.equal(call(B, e)["o"], ref)
    assert torch.equal(call(B, dict(e, block_table=torch.full((3, 2), 5, dtype=torch.int32, device="cuda")))["o"], ref)


def test_many_sequences_and_pieces_that_begin_everywhere(B):
    """More items than CTAs, and lengths that put the pieces' ends on, before and behind the items' ends."""
    d = make(22, 150, 2, 4, 4, 64, 64, [(37 * i) % 513 for i in range(150)], torch.float16)
    r = call(B, d, want_lse=True)
    check(r["o"], d, lse=r["lse"])
    d = make(23, 37, 3, 2, 2, 128, 32, [128] * 37, torch.bfloat16)
    check(call(B, d)["o"], d)


def test_views(B):
    """Queries, keys and values of one projection, a cache with the heads before the positions, an output inside a larger one."""
    d = make(7, 2, 6, 8, 2, 64, 16, [100, 40], torch.float16)
    ref = call(B, d)["o"]
    qkv = torch.cat([d["q"], d["k_new"], d["v_new"]], dim=2)
    both = torch.stack([d["k_cache"], d["v_cache"]]).transpose(2, 3).contiguous().transpose(2, 3)
    big = torch.full((2, 6, 11, 72), 4.0, dtype=torch.float16, device="cuda")
    v = dict(d, q=qkv[:, :, :8], k_new=qkv[:, :, 8:10], v_new=qkv[:, :, 10:], k_cache=both[0], v_cache=both[1])
    o = big[:, :, 2:10, :64]
    o.copy_(torch.zeros_like(o))
    call(B, v, out={"o": o})
    assert torch.equal(o, ref) and (big[:, :, :2] == 4).all() and (big[:, :, 10:] == 4).all() and (big[..., 64:] == 4).all()
    wide = torch.full((2, d["block_table"].shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, : d["block_table"].shape[1]] = d["block_table"]
    assert torch.equal(call(B, dict(d, block_table=wide[:, : d["block_table"].shape[1]]))["o"], ref)


def test_bad_pages_lengths_and_parents_are_flagged(B):
    d = make(9, 5, 4, 4, 2, 64, 16, [100, 100, 100, 100, 100], torch.bfloat16, window=2)
    d["parents"][:] = torch.tensor([0, 0, 1], dtype=torch.int32)
    good = call(B, d)["o"]
    d["block_table"][0, 3] = d["k_cache"].shape[0]
    d["block_table"][1, 0] = -1
    d["ctx_len"][2] = -4
    d["ctx_len"][3] = 16 * d["block_table"].shape[1] + 1
    d["parents"][4, 1] = 2
    flags = torch.zeros(5, dtype=torch.int32, device="cuda")
    flags[4] = 64
    out = {"o": torch.zeros_like(d["q"]), "flags": flags}
    call(B, d, out=out)
    assert flags.tolist() == [1, 1, 2, 2, 64 | 4]
    assert torch.equal(out["o"][4, [0, 1, 3]], good[4, [0, 1, 3]]) and (out["o"][4, 2] == 0).all()
    # a page that is none holds zeros
    z = dict(d, k_cache=torch.cat([d["k_cache"], torch.zeros_like(d["k_cache"][:1])]), v_cache=torch.cat([d["v_cache"], torch.zeros_like(d["v_cache"][:1])]))
    z["block_table"] = torch.where((d["block_table"] < 0) | (d["block_table"] >= d["k_cache"].shape[0]), d["k_cache"].shape[0], d["block_table"]).int()
    z["ctx_len"] = d["ctx_len"].clamp(min=0, max=16 * d["block_table"].shape[1])
    check(out["o"], z)


def test_places_beyond_32_bits(B):
    pages = (1 << 31) // (16 * 128) + 3
    kc = torch.zeros(pages, 16, 1, 128, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    kc[-2:].normal_()
    vc[-2:].normal_()
    d = make(11, 1, 3, 2, 1, 128, 16, [30], torch.bfloat16)
    d["k_cache"], d["v_cache"] = kc, vc
    d["block_table"] = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    r = call(B, d)["o"]
    small = dict(d, k_cache=kc[-2:].clone(), v_cache=vc[-2:].clone(), block_table=torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    check(r, small)


def test_the_same_bits_again_stream_graph_workspace(B):
    """Two calls, another stream, a replayed graph, a workspace full of garbage and one that two graphs share: the same bits."""
    d = make(13, 3, 21, 8, 2, 128, 16, [900, 17, 3000], torch.bfloat16)
    ref = call(B, d)["o"]
    assert torch.equal(call(B, d)["o"], ref)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    assert torch.equal(call(B, d, stream=s)["o"], ref)
    ws = torch.full((B.dssd_tree_attention_workspace_bytes(3, 21, 8, 2, 128),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(call(B, d, workspace=ws)["o"], ref)
    d2 = make(14, 3, 21, 8, 2, 128, 16, [10, 2000, 700], torch.bfloat16)
    ref2 = call(B, d2)["o"]
    outs, graphs = [], []
    for x in (d, d2):
        out = {"o": torch.zeros_like(ref), "flags": torch.zeros(3, dtype=torch.int32, device="cuda")}
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.dssd_tree_attention(*[x[k] for k in ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")], parents=x["parents"], out=out, workspace=ws)
        outs.append(out)
        graphs.append(g)
    for _ in range(2):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0]["o"], ref) and torch.equal(outs[1]["o"], ref2)
