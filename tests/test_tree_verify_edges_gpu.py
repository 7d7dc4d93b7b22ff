"""dssd_tree_verify where its arithmetic has least room: drafts that are nearly certain, siblings that exhaust them, subnormal entries, rows far
from zero, temperatures near zero.  Against the definition in float64."""
import numpy as np
import pytest
import torch

import tree_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2507_12000_b200 import binding

    return binding


def call(B, d, T, replacement):
    r = B.dssd_tree_verify(d["target_logits"], d["draft_q"], d["draft_tokens"], d["parents"], d["uniforms"], d["uniforms_rs"], T, replacement=replacement)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy().astype(np.int64) for k, v in r.items()}


def same(got, ref):
    for k in ("accept_len", "path", "token", "edge_flags", "rs_flags"):
        assert (got[k] == ref[k]).all(), (k, np.argwhere(got[k] != ref[k])[:6], got[k][:40], ref[k][:40])


def siblings(x, q, tokens, u, u_rs):
    """Sequences of one node with the listed children: x, q [V] or [B, V]; tokens, u [B, k]; u_rs [B]."""
    nb, k = np.shape(tokens)
    row = lambda a: torch.as_tensor(a).expand(nb, k + 1, -1).contiguous().cuda() if torch.as_tensor(a).dim() == 1 else torch.as_tensor(a)[:, None].expand(-1, k + 1, -1).contiguous().cuda()  # noqa: E731
    f = lambda a, t: torch.as_tensor(np.ascontiguousarray(a), dtype=t).cuda()  # noqa: E731
    return {"target_logits": row(x), "draft_q": row(q), "draft_tokens": f(tokens, torch.int32), "parents": torch.zeros(nb, k, dtype=torch.int32, device="cuda"),
            "uniforms": f(u, torch.float32), "uniforms_rs": f(u_rs, torch.float32)}


def uniforms(rng, *shape):
    return (rng.integers(0, 1 << 24, shape) * 2.0 ** -24).astype(np.float32)


@pytest.mark.parametrize("last", ["out of range", "masked in the target", "again"])
def test_a_refused_sibling_after_the_draft_is_exhausted(B, last):
    """Three siblings take all of q, a fourth is refused too: nothing is subtracted any more where q is zero."""
    V, nb = 700, 24
    rng = np.random.default_rng(4)
    x = torch.zeros(V)
    x[5] = float("-inf")
    q = torch.zeros(V)
    q[:3] = torch.tensor([0.5, 0.25, 0.25])
    tok = np.tile([0, 1, 2, {"out of range": V, "masked in the target": 5, "again": 1}[last]], (nb, 1))
    d = siblings(x, q, tok, np.full((nb, 4), 0.9), uniforms(rng, nb))
    got = call(B, d, 1.0, False)
    same(got, R.verify(d, 1.0, False))
    assert (got["rs_flags"] == 0).all() and (got["token"] >= 3).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_draft_of_subnormal_numbers(B, dtype):
    """After the one sibling of ordinary size the rest of q is subnormal in float32, and counts all the same."""
    V, nb = 300, 200
    rng = np.random.default_rng(6)
    x = torch.from_numpy(rng.normal(0, 1, V)).to(dtype)
    q = np.zeros(V, np.float32)
    q[1:41] = rng.integers(1, 90000, 40).astype(np.float32) * np.float32(2.0 ** -149)
    q[0] = 1.0
    tok = np.stack([np.zeros(nb, np.int64), rng.integers(1, 41, nb), rng.integers(1, 41, nb)], axis=1)
    d = siblings(x, torch.from_numpy(q), tok, np.concatenate([np.full((nb, 1), 0.999), uniforms(rng, nb, 2)], axis=1), uniforms(rng, nb))
    same(call(B, d, 0.9, False), R.verify(d, 0.9, False))


@pytest.mark.parametrize("gap", [9.0, 14.0, 17.0, 19.0, 30.0])
@pytest.mark.parametrize("V,dtype", [(5, torch.float32), (3001, torch.bfloat16)])
def test_siblings_of_a_draft_that_is_nearly_certain(B, gap, V, dtype):
    """Nearly all of q is one token's.  Once that is refused, the others are drawn from what is left: tails of 1e-4 to 1e-13, next to a q that
    rounds to 1."""
    nb = 600
    rng = np.random.default_rng(int(gap) * 10 + V)
    top = V // 2
    x = torch.from_numpy(rng.normal(0, 1.0, V))
    x[top] += np.log(V)
    x = x.to(dtype)
    z = rng.normal(0, 1.5, V)
    z[top] = z.max() + gap
    q = np.exp(z - z.max())
    q = torch.from_numpy((q / q.sum()).astype(np.float32))
    w = q.double().expand(nb, V).clone()
    w[:, top] = 0
    others = torch.multinomial(w, min(V - 1, 3), replacement=False, generator=torch.Generator().manual_seed(V)).numpy()
    tok = np.concatenate([np.full((nb, 1), top), others], axis=1)
    u = uniforms(rng, *tok.shape)
    u[: nb // 2, 0] = 0.999  # (as a rule refused)
    d = siblings(x, q, tok, u, uniforms(rng, nb))
    ref = R.verify(d, 0.9, False)
    same(call(B, d, 0.9, False), ref)
    assert len(np.unique(ref["path"][:, 1])) > 3


@pytest.mark.parametrize("gap", [14.0, 17.0, 19.0])
def test_the_first_token_follows_the_target_after_a_certain_draft(B, gap):
    nb = 1 << 17
    p = np.array([0.6, 0.2, 0.1, 0.06, 0.04])
    z = np.array([0.0, -gap, -gap - 0.4, -gap - 0.2, -gap - 1.0])
    q = torch.softmax(torch.from_numpy(z), 0).float()
    gen = torch.Generator(device="cuda").manual_seed(int(gap))
    tok = torch.multinomial(q.double().cuda().expand(nb, 5), 2, replacement=False, generator=gen)
    d = {"target_logits": torch.log(torch.from_numpy(p)).float().cuda().expand(nb, 3, 5).contiguous(), "draft_q": q.cuda().expand(nb, 3, 5).contiguous(),
         "draft_tokens": tok.int(), "parents": torch.zeros(nb, 2, dtype=torch.int32, device="cuda"), "uniforms": torch.rand(nb, 2, generator=gen, device="cuda"),
         "uniforms_rs": torch.rand(nb, generator=gen, device="cuda")}
    r = call(B, d, 1.0, False)
    first = np.where(r["accept_len"] == 1, np.take_along_axis(tok.cpu().numpy(), np.maximum(r["path"][:, 1:2] - 1, 0), 1)[:, 0], r["token"])
    freq = np.bincount(first, minlength=5) / nb
    # five standard deviations of a frequency of nb draws, as in the test of drafts that are not certain
    assert (np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / nb)).all(), (freq, p)


def test_the_same_sibling_twice(B):
    """A token that was refused has left q: once more among the siblings it changes nothing."""
    rng = np.random.default_rng(12)
    V, nb = 900, 300
    x = torch.from_numpy(rng.normal(0, 1.5, V)).float()
    q = torch.softmax(x + torch.from_numpy(rng.normal(0, 1.0, V)).float(), 0)
    a = torch.multinomial(q, nb, replacement=True, generator=torch.Generator().manual_seed(3)).numpy()
    b = torch.multinomial(q, nb, replacement=True, generator=torch.Generator().manual_seed(4)).numpy()
    d = siblings(x, q, np.stack([a, a, b, a], axis=1), uniforms(rng, nb, 4), uniforms(rng, nb))
    same(call(B, d, 1.0, False), R.verify(d, 1.0, False))


def test_many_siblings_without_replacement(B):
    """More refused siblings than a warp has lanes, all over the row and several to a block."""
    rng = np.random.default_rng(14)
    for V, dtype in ((2500, torch.bfloat16), (130, torch.float32)):
        nb, k = 12, 60
        x = torch.from_numpy(rng.normal(0, 1.0, (nb, V))).to(dtype)
        x[:, ::2] -= 12  # (refused as a rule)
        q = np.exp(rng.normal(0, 1.0, (nb, V)) - 6.0 * (np.arange(V) % 2))
        q = torch.from_numpy((q / q.sum(axis=1, keepdims=True)).astype(np.float32))
        tok = torch.multinomial(q.double(), k, replacement=False, generator=torch.Generator().manual_seed(V)).numpy()
        d = siblings(x, q, tok, 0.5 + 0.5 * uniforms(rng, nb, k), uniforms(rng, nb))
        ref = R.verify(d, 1.0, False)
        same(call(B, d, 1.0, False), ref)
        assert (ref["path"][:, 1] > 33).any() or (ref["accept_len"] == 0).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1.0, 0.37, 1e30, 1e-9, 1e-18])
def test_rows_far_from_zero(B, dtype, T):
    """Rows that hold nothing above their type's lowest value, in part or altogether, and rows of 1e30: what counts is the distance from
    the largest entry."""
    rng = np.random.default_rng(23)
    d = R.verify_inputs(rng, 9, 4, 600, dtype, window=2, ragged=False)
    low, x = torch.finfo(dtype).min, d["target_logits"]
    x[0] = low
    x[1] = low
    x[1, :, ::3] = float("-inf")
    x[2] = low
    x[2, :, 7] = low / 2
    x[3] = 1e30
    x[4, :, ::2] = 1e30
    x[5, :, 1::2] = -1e30
    x[6] = -1e30
    x[7, :, 300:] = torch.finfo(dtype).max
    same(call(B, d, T, True), R.verify(d, T, True))


@pytest.mark.parametrize("T", [1e-4, 1e-6, 1e-9, 1e-12, 1e-15])
def test_temperatures_near_zero(B, T):
    """One entry above zeros: at these temperatures it has all of the mass, wherever the rounding of its scaled value falls."""
    rng = np.random.default_rng(2)
    nb, V = 256, 900
    x = torch.zeros(nb, V)
    at = rng.integers(0, V, nb)
    x[torch.arange(nb), torch.from_numpy(at)] = torch.from_numpy(rng.uniform(1.0, 60.0, nb)).float()
    q = torch.full((nb, V), 1.0 / V)
    d = siblings(x, q, rng.integers(0, V, (nb, 2)), uniforms(rng, nb, 2), uniforms(rng, nb))
    got = call(B, d, T, True)
    same(got, R.verify(d, T, True))
    assert ((got["token"] == at) | (got["accept_len"] == 1)).all()


@pytest.mark.parametrize("bits", [60, 90, 115])
def test_decisions_on_tokens_far_down(B, bits):
    """A token of 2^-60 to 2^-115 of the mass, with uniforms within float32's errors of its test's edge.  (T = 1.44: the rounding of
    log2(e)/T weighs most just above 1.)"""
    nb, V = 512, 6
    rng = np.random.default_rng(bits)
    T = 1.4426950408889634 / (1.0 + rng.uniform(0, 1, nb) * 2.0 ** -6)
    bad = []
    for b in range(0, nb, 8):  # one temperature to a call
        t = float(T[b])
        x = np.zeros((8, V), np.float32)
        x[:, 3] = -(bits + rng.uniform(0, 1, 8)) * np.log(2.0) * t
        p = np.exp(x[:, 3].astype(np.float64) / t) / np.exp(x.astype(np.float64) / t).sum(axis=1)
        q = np.full((8, V), 0.2, np.float32)
        q[:, 3] = (p * rng.uniform(1.2, 1.9, 8)).astype(np.float32)
        u = (p / q[:, 3].astype(np.float64) * (1 + np.array([-5, -3, -2, -1, 1, 2, 3, 5]) * 1e-6)).astype(np.float32)
        d = siblings(torch.from_numpy(x), torch.from_numpy(q), np.full((8, 1), 3), u[:, None], uniforms(rng, 8))
        got, ref = call(B, d, t, True), R.verify(d, t, True)
        if (got["accept_len"] != ref["accept_len"]).any():
            bad.append((b, got["accept_len"], ref["accept_len"]))
    assert not bad, (len(bad), bad[:4])
