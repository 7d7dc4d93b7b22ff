"""Rounds on drafted trees as a serving loop runs them: attention over the cache, adjusted logits, the verdict, the path into the
cache, and the next round on what this one left.  The state is checked against definitions in float64 at every step."""
import numpy as np
import pytest
import torch

import tree_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,replacement", [(torch.bfloat16, True), (torch.float16, False)])
def test_rounds_follow_one_another(dtype, replacement):
    from paper_2507_12000_b200 import binding as B
    from paper_2507_12000_b200.tree import verify_round_tree

    rng = np.random.default_rng(5)
    gen = torch.Generator(device="cuda").manual_seed(5)
    nb, N, V, layers, Hq, Hkv, D, page, T = 5, 12, 700, 2, 8, 2, 64, 8, 0.9
    # keys and values of a layer depend on the token alone, so that the cache's contents are known exactly
    k_of = torch.randn(layers, V, Hkv, D, generator=gen, device="cuda").to(dtype)
    v_of = torch.randn(layers, V, Hkv, D, generator=gen, device="cuda").to(dtype)
    q_of = torch.randn(layers, V, Hq, D, generator=gen, device="cuda").to(dtype)
    head = torch.randn(Hq * D, V, generator=gen, device="cuda") * 0.2
    per = 12
    table = torch.from_numpy(rng.permutation(nb * per + 3)[: nb * per].reshape(nb, per).astype(np.int32)).cuda()
    k_cache = torch.full((layers, nb * per + 3, page, Hkv, D), float("nan"), dtype=dtype, device="cuda")
    v_cache = k_cache.clone()
    text = [list(rng.integers(0, V, int(rng.integers(1, 9)))) for _ in range(nb)]  # the last token is not in the cache yet
    L = 80
    # the prompts, but for their last tokens, by one call
    longest = max(len(x) for x in text)
    rows = torch.zeros(nb, longest, dtype=torch.long, device="cuda")
    for b, x in enumerate(text):
        rows[b, : len(x)] = torch.tensor(x)
    ctx = torch.zeros(nb, dtype=torch.int32, device="cuda")
    first = torch.tensor([len(x) - 2 for x in text], dtype=torch.int32, device="cuda")
    ctx = B.dssd_cache_append(k_of[:, rows], v_of[:, rows], k_cache, v_cache, table, ctx, first)["new_len"]
    prompt = torch.tensor([len(x) for x in text], dtype=torch.int32, device="cuda")
    flags = torch.zeros(nb, dtype=torch.int32, device="cuda")
    accepted = 0
    for step in range(5):
        parents = torch.from_numpy(R.random_parents(rng, nb, N, window=3)).cuda()
        root = torch.tensor([[x[-1]] for x in text], device="cuda")
        par = parents.long().clamp(min=0)
        # the draft: a noisy guess at every node's row, children drawn from it
        o = [None] * layers
        draft = torch.zeros(nb, N - 1, dtype=torch.int32, device="cuda")
        guess = torch.softmax(torch.randn(nb, N, V, generator=gen, device="cuda"), dim=-1)
        if replacement:
            draft = torch.multinomial(guess.reshape(nb * N, V), N, replacement=True, generator=gen).reshape(nb, N, N)
        else:
            draft = torch.multinomial(guess.reshape(nb * N, V), N, generator=gen).reshape(nb, N, N)
        place = torch.tril((par[:, :, None] == par[:, None, :]) & (parents >= 0)[:, None, :], diagonal=-1).sum(dim=2)
        draft = draft[torch.arange(nb, device="cuda")[:, None], par, place].int()
        nodes = torch.cat([root, draft.long()], dim=1)
        # the target model: attention layers, then logits near the draft's so that some tokens are accepted
        for l in range(layers):
            d = {"q": q_of[l][nodes], "k_new": k_of[l][nodes], "v_new": v_of[l][nodes], "k_cache": k_cache[l], "v_cache": v_cache[l],
                 "block_table": table, "ctx_len": ctx, "parents": parents}
            o[l] = B.dssd_tree_attention(*[d[k] for k in ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")], parents=parents,
                                         out={"o": torch.zeros_like(d["q"]), "flags": flags})["o"]
            ref, _, live, wv, big = R.attention(dict(d, k_cache=torch.nan_to_num(k_cache[l]), v_cache=torch.nan_to_num(v_cache[l])), D ** -0.5)
            eps = R.EPS[dtype]
            tol = (eps + 4 * D * 2.0 ** -24 * big[..., None] + 2.0 ** -20) * wv + eps * np.abs(ref) * 1.01 + (100 * 2.0 ** -25 * 6 if dtype == torch.float16 else 0)
            assert (np.abs(R.f64(o[l]) - ref) <= tol)[live].all()
        logits = (o[-1].float().reshape(nb, N, Hq * D) @ head + torch.log(guess) * T).contiguous()
        history = torch.zeros(nb, L, dtype=torch.int32, device="cuda")
        for b, x in enumerate(text):
            history[b, : len(x)] = torch.tensor(x, dtype=torch.int32)
        adjust = {"history": history, "prompt_len": prompt, "history_len": torch.tensor([len(x) for x in text], dtype=torch.int32, device="cuda"),
                  "repetition": torch.full((nb,), 1.1, device="cuda"), "frequency": torch.full((nb,), 0.2, device="cuda"),
                  "mask": torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (3, (V + 31) // 32)).astype(np.int32) | 0x55555555).cuda(),
                  "mask_row": torch.from_numpy(rng.integers(-1, 3, (nb, N)).astype(np.int32)).cuda()}
        expect, mag, live, _ = R.adjust(dict(adjust, logits=logits, draft_tokens=draft, parents=parents))
        uni = {"uniforms": torch.rand(nb, N - 1, generator=gen, device="cuda"), "uniforms_rs": torch.rand(nb, generator=gen, device="cuda")}
        r = verify_round_tree(logits, guess.contiguous(), draft, parents, uni["uniforms"], uni["uniforms_rs"], T, replacement=replacement, adjust=adjust,
                              cache={"k_new": k_of[:, nodes], "v_new": v_of[:, nodes], "k_cache": k_cache, "v_cache": v_cache, "block_table": table, "ctx_len": ctx})
        torch.cuda.synchronize()
        got = R.f64(logits)
        with np.errstate(invalid="ignore"):
            fine = (got == expect) | (np.abs(got - expect) <= 2.0 ** -24 * np.abs(expect) + 5 * 2.0 ** -24 * mag)
        assert fine[live].all()
        ref = R.verify({"target_logits": logits, "draft_q": guess, "draft_tokens": draft, "parents": parents, **uni}, T, replacement)
        for k in ("accept_len", "path", "token", "edge_flags", "rs_flags"):
            assert (r[k].cpu().numpy() == ref[k]).all(), (step, k)
        assert (r["adjust_flags"] == 0).all() and (r["cache_flags"] == 0).all() and (flags == 0).all()
        for b in range(nb):
            way = [int(draft[b, j - 1]) for j in ref["path"][b][1:] if j > 0]
            new = way + [int(ref["token"][b])]
            assert r["tokens"][b].tolist() == new + [-1] * (N - len(new))
            text[b] += new
            accepted += len(way)
        ctx = r["new_len"]
        # the cache holds all tokens but the last, and NaN elsewhere
        for b, x in enumerate(text):
            assert int(ctx[b]) == len(x) - 1
            pos = torch.arange(len(x) - 1, device="cuda")
            t = torch.tensor(x[:-1], device="cuda")
            pg, of = table[b].long()[pos // page], pos % page
            assert torch.equal(k_cache[:, pg, of], k_of[:, t]) and torch.equal(v_cache[:, pg, of], v_of[:, t])
        assert int(torch.isfinite(k_cache[0, :, :, 0, 0]).sum()) == sum(len(x) - 1 for x in text)
    assert accepted > 0  # some drafted tokens went into the cache with the roots


def test_a_round_is_captured():
    """A whole round in a CUDA graph gives what the calls give one by one."""
    from paper_2507_12000_b200.tree import verify_round_tree

    rng = np.random.default_rng(9)
    d = R.verify_inputs(rng, 4, 9, 2000, torch.float32, T=0.8)
    kv = {"k_new": torch.randn(3, 4, 9, 2, 16, device="cuda").half(), "v_new": torch.randn(3, 4, 9, 2, 16, device="cuda").half(),
          "k_cache": torch.zeros(3, 9, 16, 2, 16, device="cuda").half(), "v_cache": torch.zeros(3, 9, 16, 2, 16, device="cuda").half(),
          "block_table": torch.arange(8, dtype=torch.int32, device="cuda").reshape(4, 2), "ctx_len": torch.tensor([0, 5, 16, 20], dtype=torch.int32, device="cuda")}
    adjust = {"bias_tokens": torch.tensor([[3], [4], [5], [6]], dtype=torch.int32, device="cuda"), "bias_values": torch.full((4, 1), 9.0, device="cuda")}
    args = (d["draft_q"], d["draft_tokens"], d["parents"], d["uniforms"], d["uniforms_rs"], 0.8)
    start = d["target_logits"].clone()
    one = verify_round_tree(d["target_logits"], *args, adjust=adjust, cache=kv)
    k_one, logits_one = kv["k_cache"].clone(), d["target_logits"].clone()
    g = torch.cuda.CUDAGraph()
    work = start.clone()
    kv["k_cache"].zero_()
    with torch.cuda.graph(g):
        two = verify_round_tree(work, *args, adjust=adjust, cache=kv)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(one[k], two[k]) for k in one)
    assert torch.equal(work, logits_one) and torch.equal(kv["k_cache"], k_one)
