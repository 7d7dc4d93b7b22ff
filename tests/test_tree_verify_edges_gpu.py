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
