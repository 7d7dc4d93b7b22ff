"""Performance cases of the operators around a verification round: logits made ready for the verdict, the
target model's attention for a tree of drafted tokens, the verdict on that tree, and the cache that keeps
what was accepted.

`run` computes an operator in its plain form (elementary torch operations) or, where `own` is true, through
the library's entry points.

Operators:
  adjust   dssd_adjust_logits   penalties for repeated tokens, biases and grammar masks
  attend   dssd_tree_attention  attention of a tree of drafted tokens over a paged cache
  verify   dssd_tree_verify     the verdict on a drafted tree and the token drawn after it
  append   dssd_cache_append    keys and values of the accepted path into the pages

A tree of N nodes: node 0 is the root (the last committed token), node j = 1 .. N-1 holds drafted token j-1
and hangs under node parents[j-1] < j; a negative parent marks a place without a node.
"""
from __future__ import annotations

import math
from typing import Dict

import torch

own = False

MAX_ROW_BYTES = 1 << 30      # logits of the largest batch (and their copy)
MAX_DRAFT_BYTES = 5 << 28    # draft rows of the largest batch
MAX_CACHE_BYTES = 3 << 29    # keys and values of the largest batch
MAX_ATTEND_FLOPS = 6e11
MAX_SCORE_BYTES = 3 << 30    # what the plain form of the attention holds of scores


def _adjust(batch, rows, vocab, dtype, history, window=0, penalties=True, masked=0.0, in_place=False, name=""):
    return _named({"op": "adjust", "B": batch, "N": rows, "V": vocab, "dtype": dtype, "L": history, "window": window,
                   "penalties": penalties, "masked": masked, "in_place": in_place}, name)


def _attend(batch, nodes, hq, hkv, dim, ctx, page, dtype, window=0, ragged=True, name=""):
    return _named({"op": "attend", "B": batch, "N": nodes, "Hq": hq, "Hkv": hkv, "D": dim, "ctx": ctx, "page": page,
                   "dtype": dtype, "window": window, "ragged": ragged}, name)


def _verify(batch, nodes, vocab, dtype, T, sigma_d, window, replacement, name=""):
    return _named({"op": "verify", "B": batch, "N": nodes, "V": vocab, "dtype": dtype, "T": T, "sigma_d": sigma_d,
                   "window": window, "replacement": replacement}, name)


def _append(layers, batch, nodes, hkv, dim, page, path, dtype, name=""):
    return _named({"op": "append", "layers": layers, "B": batch, "N": nodes, "Hkv": hkv, "D": dim, "page": page,
                   "path": path, "dtype": dtype}, name)


def _named(case: Dict, name: str) -> Dict:
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one user, eight drafted tokens in a chain: what the logits wait for before the verdict
        _adjust(1, 9, 50272, "f32", 600, name="adjust_B1_N9_V50272_f32"),
        # an ordinary batch of drafted trees, ragged, a few requests under a grammar; a fresh copy is wanted
        _adjust(32, 24, 128256, "bf16", 2000, window=6, masked=0.25, name="adjust_B32_N24_V128256_bf16"),
        # a large batch of short drafts, in place: only what a request asks for is touched
        _adjust(256, 5, 151936, "bf16", 1500, penalties=False, masked=0.1, in_place=True, name="adjust_B256_N5_V151936_bf16_in"),
        # one user, one token: the latency of a decoding step over a short cache
        _attend(1, 1, 32, 8, 128, 2047, 16, "bf16", ragged=False, name="attend_B1_N1_ctx2047_bf16"),
        # an ordinary batch, chains of four drafted tokens, ragged contexts, seven query heads to a key head
        _attend(32, 5, 28, 4, 128, 6000, 16, "bf16", name="attend_B32_N5_G7_ctx6000_bf16"),
        # trees of 64 nodes in a batch, eight query heads to a key head
        _attend(8, 64, 64, 8, 128, 8000, 64, "bf16", window=16, name="attend_B8_N64_G8_ctx8000_bf16"),
        # one long document and a tree
        _attend(1, 32, 32, 8, 128, 131071, 32, "f16", window=10, ragged=False, name="attend_B1_N32_ctx131071_f16"),
        # the verdict for one user: latency
        _verify(1, 16, 50272, "f32", 1.0, 0.6, 4, True, name="verify_B1_N16_V50272_f32"),
        # distinct siblings (drawn without replacement), often rejected
        _verify(48, 32, 32000, "bf16", 0.8, 1.0, 8, False, name="verify_B48_N32_V32000_bf16"),
        # a large batch
        _verify(128, 12, 151936, "bf16", 0.7, 0.7, 4, True, name="verify_B128_N12_V151936_bf16"),
        # the accepted paths of a batch into all layers' pages
        _append(32, 64, 16, 8, 128, 16, True, "bf16", name="append_L32_B64_N16_bf16"),
        # one layer of a prompt, as a model's prefill writes it
        _append(1, 4, 1500, 8, 128, 16, False, "bf16", name="append_L1_B4_N1500_bf16"),
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _vocab(rng) -> int:
    v = _log_int(rng, 1024, 160000)
    return (v + 15) // 16 * 16 if rng.random() < 0.6 else v


def draw(rng):
    op = rng.choice(["adjust", "attend", "attend", "verify", "append"])
    while True:
        if op == "adjust":
            c = _adjust(_log_int(rng, 1, 256), _log_int(rng, 1, 48), _vocab(rng), rng.choice(["bf16", "f32"]),
                        _log_int(rng, 1, 20000), rng.choice([0, 0, 4, 9]), rng.random() < 0.7, rng.choice([0.0, 0.2, 0.7]))
            c["in_place"] = not c["penalties"] and rng.random() < 0.5
            if c["B"] * c["N"] * c["V"] * _size(c) <= MAX_ROW_BYTES // 5 and c["B"] * c["L"] <= 1 << 21:
                return c
        elif op == "attend":
            hkv, g = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16])
            c = _attend(_log_int(rng, 1, 64), _log_int(rng, 1, 96), hkv * g, hkv, rng.choice([64, 96, 128, 128]),
                        _log_int(rng, 16, 100000), rng.choice([8, 16, 32, 48, 64, 256]), rng.choice(["bf16", "f16"]),
                        rng.choice([0, 5, 16]), rng.random() < 0.7)
            w = work(c)
            if (w["bytes"] <= MAX_CACHE_BYTES // 4 and w["flops"] <= MAX_ATTEND_FLOPS / 8
                    and 4 * c["B"] * c["Hq"] * c["N"] * c["ctx"] <= MAX_SCORE_BYTES // 2):
                return c
        elif op == "verify":
            c = _verify(_log_int(rng, 1, 160), _log_int(rng, 1, 48), _vocab(rng), rng.choice(["bf16", "f32"]),
                        rng.choice([0.6, 0.8, 1.0, 1.2]), round(rng.uniform(0.2, 1.2), 2), rng.choice([1, 4, 9]),
                        rng.random() < 0.5)
            if c["B"] * c["N"] * c["V"] * 4 <= MAX_DRAFT_BYTES // 2:
                return c
        else:
            c = _append(_log_int(rng, 1, 40), _log_int(rng, 1, 96), _log_int(rng, 1, 300), rng.choice([1, 2, 4, 8]),
                        rng.choice([64, 96, 128]), rng.choice([8, 16, 48, 64]), rng.random() < 0.5,
                        rng.choice(["bf16", "f16"]))
            if c["layers"] * c["B"] * (c["N"] + 100) * c["Hkv"] * c["D"] * 4 <= 1 << 30:
                return c


def _size(case) -> int:
    return 4 if case["dtype"] == "f32" else 2


def _type(case) -> torch.dtype:
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[case["dtype"]]


# ---- inputs ----------------------------------------------------------------------------------


def _gen(seed: int) -> torch.Generator:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _uniform(shape, gen) -> torch.Tensor:
    """Multiples of 2^-24 in [0, 1)."""
    return torch.randint(0, 1 << 24, shape, generator=gen, device="cuda").to(torch.float32) * 2.0 ** -24


def _tree(nb: int, n: int, window: int, gen):
    """parents [B, N-1]: every node hangs under one of the `window` nodes before it; the batch is ragged: some
    sequences have fewer nodes.  window 0: chains of full length."""
    j = torch.arange(1, n, device="cuda")
    if window == 0:
        return (j - 1).expand(nb, n - 1).to(torch.int32).contiguous()
    back = torch.minimum((torch.rand(nb, n - 1, generator=gen, device="cuda") * window).long(), j - 1)
    count = torch.randint((n + 1) // 2, n + 1, (nb, 1), generator=gen, device="cuda")
    return torch.where(j < count, j - 1 - back, torch.full_like(back, -1)).to(torch.int32)


def _logits(nb, n, V, dtype, gen):
    """Gaussian logits over a Zipf(1.1) bias, as the workload generator of the benchmark makes them."""
    beta = -1.1 * torch.log1p(torch.randperm(V, generator=gen, device="cuda").to(torch.float32))
    out = torch.empty(nb, n, V, dtype=dtype, device="cuda")
    for b in range(0, nb, max(1, (1 << 26) // (n * V))):
        e = min(nb, b + max(1, (1 << 26) // (n * V)))
        out[b:e] = torch.randn(e - b, n, V, generator=gen, device="cuda").mul_(3.0).add_(beta)
    return out, beta


def _prepare_adjust(c, seed):
    nb, n, V, L, gen = c["B"], c["N"], c["V"], c["L"], _gen(seed)
    logits, beta = _logits(nb, n, V, _type(c), gen)
    order = torch.argsort(beta, descending=True)
    # tokens of a text: ranks of a power law, so that some repeat often and many come once
    rank = (V ** torch.rand(nb, L + n, generator=gen, device="cuda", dtype=torch.float64)).long().clamp_(max=V) - 1
    text = order[rank].to(torch.int32)
    length = torch.randint((L + 1) // 2, L + 1, (nb,), generator=gen, device="cuda", dtype=torch.int32)
    s = {"case": dict(c), "logits": logits, "history": text[:, :L].contiguous(), "history_len": length,
         "prompt_len": (length * torch.rand(nb, generator=gen, device="cuda")).to(torch.int32),
         "draft_tokens": text[:, L:L + n - 1].contiguous(), "parents": None}
    if c["window"]:
        s["parents"] = _tree(nb, n, c["window"], gen)
    one = torch.rand(nb, generator=gen, device="cuda")
    s["repetition"] = 1.0 + 0.3 * one if c["penalties"] else None
    s["presence"] = torch.rand(nb, generator=gen, device="cuda")
    s["frequency"] = 0.5 * torch.rand(nb, generator=gen, device="cuda")
    k = min(32, V)
    s["bias_tokens"] = torch.rand(nb, V, generator=gen, device="cuda").topk(k, dim=1).indices.to(torch.int32)
    s["bias_tokens"][:, k // 2:][torch.rand(nb, k - k // 2, generator=gen, device="cuda") < 0.5] = -1
    s["bias_values"] = 5.0 * torch.randn(nb, k, generator=gen, device="cuda")
    s["mask"] = s["mask_row"] = None
    if c["masked"]:
        # a grammar for some of the requests: a state of it allows a handful of tokens or most of them
        under = torch.rand(nb, 1, generator=gen, device="cuda") < c["masked"]
        states, words = 64, (V + 31) // 32
        few = torch.randint(-2 ** 31, 2 ** 31, (3, states, words), generator=gen, device="cuda")
        few = few[0] & few[1] & few[2]
        few[: states // 2] &= torch.randint(0, 64, (states // 2, words), generator=gen, device="cuda") // 63 * -1
        s["mask"] = few.to(torch.int32)
        state = torch.randint(0, states, (nb, n), generator=gen, device="cuda", dtype=torch.int32)
        s["mask_row"] = torch.where(under, state, torch.full_like(state, -1))
    s["out"] = {"logits": logits if c["in_place"] else torch.zeros_like(logits),
                "flags": torch.zeros(nb, dtype=torch.int32, device="cuda")}
    return s


def _lengths(c, gen):
    if not c["ragged"]:
        return torch.full((c["B"],), c["ctx"], dtype=torch.int32, device="cuda")
    return torch.randint(max(0, c["ctx"] // 8), c["ctx"] + 1, (c["B"],), generator=gen, device="cuda", dtype=torch.int32)


def _prepare_attend(c, seed):
    nb, n, dt, gen = c["B"], c["N"], _type(c), _gen(seed)
    length = _lengths(c, gen)
    per = max(1, -(-c["ctx"] // c["page"]))
    # pages handed out in any order, with some that belong to nobody here
    total = nb * per + 3
    table = torch.randperm(total, generator=gen, device="cuda")[: nb * per].reshape(nb, per).to(torch.int32)

    def rows(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float16)).to(dt)

    return {"case": dict(c), "q": rows(nb, n, c["Hq"], c["D"], scale=1.5), "k_new": rows(nb, n, c["Hkv"], c["D"]),
            "v_new": rows(nb, n, c["Hkv"], c["D"]), "k_cache": rows(total, c["page"], c["Hkv"], c["D"]),
            "v_cache": rows(total, c["page"], c["Hkv"], c["D"]), "block_table": table, "ctx_len": length,
            "parents": _tree(nb, n, c["window"], gen) if c["window"] and n > 1 else None,
            "out": {"o": torch.zeros(nb, n, c["Hq"], c["D"], dtype=dt, device="cuda"),
                    "flags": torch.zeros(nb, dtype=torch.int32, device="cuda")}}


def _prepare_verify(c, seed):
    nb, n, V, gen = c["B"], c["N"], c["V"], _gen(seed)
    s = {"case": dict(c), "parents": _tree(nb, n, c["window"], gen)}
    s["target_logits"], _ = _logits(nb, n, V, _type(c), gen)
    s["draft_q"] = torch.empty(nb, n, V, device="cuda")
    s["draft_tokens"] = torch.zeros(nb, max(0, n - 1), dtype=torch.int32, device="cuda")
    par = s["parents"].long().clamp(min=0)
    # a node's place among its siblings
    same = (par[:, :, None] == par[:, None, :]) & (s["parents"] >= 0)[:, None, :]
    place = torch.tril(same, diagonal=-1).sum(dim=2)
    most = min(V, 64)
    step = max(1, (1 << 26) // (n * V))
    for b in range(0, nb, step):
        e = min(nb, b + step)
        q = torch.randn(e - b, n, V, generator=gen, device="cuda").mul_(c["sigma_d"]).add_(s["target_logits"][b:e]).div_(c["T"])
        q = torch.softmax(q, dim=-1)
        s["draft_q"][b:e] = q
        if n > 1:
            r = par[b:e]
            if c["replacement"]:
                cdf = torch.cumsum(q, dim=-1).gather(1, r[:, :, None].expand(-1, -1, V))
                u = torch.rand(e - b, n - 1, 1, generator=gen, device="cuda") * cdf[:, :, -1:]
                t = torch.searchsorted(cdf, u, right=True).squeeze(2).clamp_(max=V - 1)
            else:  # exponential clocks: the order in which they ring is a draw without replacement
                ring = torch.empty_like(q).exponential_(generator=gen).div_(q.clamp(min=1e-30)).neg_()
                t = ring.topk(most, dim=-1).indices[torch.arange(e - b, device="cuda")[:, None], r, place[b:e].clamp(max=most - 1)]
            s["draft_tokens"][b:e] = t.to(torch.int32)
    s["uniforms"] = _uniform((nb, max(0, n - 1)), gen)
    s["uniforms_rs"] = _uniform((nb,), gen)
    s["out"] = {k: torch.zeros(nb, dtype=torch.int32, device="cuda") for k in ("accept_len", "token", "edge_flags", "rs_flags")}
    s["out"]["path"] = torch.zeros(nb, n, dtype=torch.int32, device="cuda")
    return s


def _prepare_append(c, seed):
    nb, n, dt, gen = c["B"], c["N"], _type(c), _gen(seed)
    length = torch.randint(0, 64, (nb,), generator=gen, device="cuda", dtype=torch.int32)
    per = -(-(64 + n) // c["page"])
    total = nb * per + 1

    def rows(*shape):
        return torch.randn(*shape, c["Hkv"], c["D"], generator=gen, device="cuda", dtype=torch.float16).to(dt)

    s = {"case": dict(c), "k_new": rows(c["layers"], nb, n), "v_new": rows(c["layers"], nb, n),
         "k_cache": rows(c["layers"], total, c["page"]), "v_cache": rows(c["layers"], total, c["page"]),
         "block_table": torch.randperm(total, generator=gen, device="cuda")[: nb * per].reshape(nb, per).to(torch.int32),
         "ctx_len": length, "path": None}
    if c["path"]:  # the root and a few nodes further on
        most = min(n, 8)
        s["accept_len"] = torch.randint(0, most, (nb,), generator=gen, device="cuda", dtype=torch.int32)
        pick = torch.rand(nb, n - 1, generator=gen, device="cuda").argsort(dim=1)[:, : most - 1].sort(dim=1).values + 1
        s["path"] = torch.full((nb, n), -1, dtype=torch.int32, device="cuda")
        s["path"][:, 0] = 0
        s["path"][:, 1:most] = pick.to(torch.int32)
        s["path"][torch.arange(n, device="cuda") > s["accept_len"][:, None]] = -1
    else:
        s["accept_len"] = torch.randint(n // 2, n, (nb,), generator=gen, device="cuda", dtype=torch.int32)
    s["out"] = {k: torch.zeros(nb, dtype=torch.int32, device="cuda") for k in ("new_len", "flags")}
    return s


def prepare(case, seed):
    return {"adjust": _prepare_adjust, "attend": _prepare_attend, "verify": _prepare_verify, "append": _prepare_append}[case["op"]](case, seed)


# ---- one pass: the library's entry points ------------------------------------------------------


def _run_own(s):
    from paper_2507_12000_b200 import binding as B

    c, op = s["case"], s["case"]["op"]
    if op == "adjust":
        return B.dssd_adjust_logits(s["logits"], s["history"], s["prompt_len"], s["history_len"], draft_tokens=s["draft_tokens"],
                                    parents=s["parents"], repetition=s["repetition"], presence=s["presence"],
                                    frequency=s["frequency"], bias_tokens=s["bias_tokens"], bias_values=s["bias_values"],
                                    mask=s["mask"], mask_row=s["mask_row"], out=s["out"])["logits"]
    if op == "attend":
        if "ws" not in s:  # kept by a serving loop for all layers and steps
            s["ws"] = torch.empty(B.dssd_tree_attention_workspace_bytes(c["B"], c["N"], c["Hq"], c["Hkv"], c["D"]),
                                  dtype=torch.uint8, device="cuda")
        return B.dssd_tree_attention(s["q"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["block_table"], s["ctx_len"],
                                     parents=s["parents"], out=s["out"], workspace=s["ws"])["o"]
    if op == "verify":
        if "ws" not in s:
            s["ws"] = torch.empty(B.dssd_tree_verify_workspace_bytes(c["B"], c["N"], c["V"]), dtype=torch.uint8, device="cuda")
        r = B.dssd_tree_verify(s["target_logits"], s["draft_q"], s["draft_tokens"], s["parents"], s["uniforms"], s["uniforms_rs"],
                               c["T"], replacement=c["replacement"], out=s["out"], workspace=s["ws"])
        return {k: r[k] for k in ("accept_len", "path", "token")}
    r = B.dssd_cache_append(s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["block_table"], s["ctx_len"], s["accept_len"],
                            path=s["path"], out=s["out"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "new_len": r["new_len"]}


# ---- one pass: the plain forms -----------------------------------------------------------------


def _ancestors(parents, nb, n):
    """[B, N, N]: node i lies on the way from the root to node j, j itself included; [B, N]: there is a node j."""
    up = torch.zeros(nb, n, n, device="cuda")
    if n > 1:
        up[:, 1:].scatter_(2, parents.long().clamp(min=0)[:, :, None], (parents >= 0).float()[:, :, None])
    reach = up + torch.eye(n, device="cuda")
    for _ in range(max(1, n).bit_length()):  # ways of up to 1, 2, 4, ... steps
        reach = (reach @ reach > 0).float()
    return reach > 0, reach[:, :, 0] > 0


def _chain(nb, n):
    return torch.arange(0, n - 1, dtype=torch.int32, device="cuda").expand(nb, n - 1)


def _plain_adjust(s):
    c = s["case"]
    nb, n, V, L = c["B"], c["N"], c["V"], c["L"]
    at = torch.arange(L, device="cuda")
    seen = (at < s["history_len"][:, None]).float()
    out = seen * (at >= s["prompt_len"][:, None])
    words = s["history"].long()
    n_all = torch.zeros(nb, V, device="cuda").scatter_add_(1, words, seen)
    n_out = torch.zeros(nb, V, device="cuda").scatter_add_(1, words, out)
    on, there = _ancestors(_chain(nb, n) if s["parents"] is None else s["parents"], nb, n)
    drafted = torch.zeros(nb, n, V, device="cuda")
    if n > 1:
        drafted.scatter_add_(2, s["draft_tokens"].long()[:, None, :].expand(nb, n, n - 1), on[:, :, 1:].float())
    x = s["logits"].float()
    if s["repetition"] is not None:
        r = s["repetition"][:, None, None]
        x = torch.where(n_all[:, None] + drafted > 0, torch.where(x > 0, x / r, x * r), x)
    n_out = drafted.add_(n_out[:, None])
    x = x - s["frequency"][:, None, None] * n_out
    x = x - s["presence"][:, None, None] * (n_out > 0)
    del n_out, drafted
    bias = torch.zeros(nb, V + 1, device="cuda")
    where = s["bias_tokens"].long()
    bias.scatter_(1, torch.where(where < 0, V, where), s["bias_values"])
    x = x + bias[:, None, :V]
    if s["mask"] is not None:
        bit = torch.arange(V, device="cuda")
        allowed = (s["mask"][:, bit // 32] >> (bit % 32)) & 1
        banned = (allowed == 0)[s["mask_row"].long().clamp(min=0)] & (s["mask_row"] >= 0)[:, :, None]
        x = x.masked_fill_(banned, -math.inf)
        del banned
    o = s["out"]["logits"]
    o.copy_(torch.where(there[:, :, None], x.to(o.dtype), o))
    return o


def _plain_attend(s):
    c = s["case"]
    nb, n, hq, hkv, D = c["B"], c["N"], c["Hq"], c["Hkv"], c["D"]
    table = s["block_table"].long()
    k = torch.cat([s["k_cache"][table].float().reshape(nb, -1, hkv, D), s["k_new"].float()], dim=1)
    ctx = k.shape[1] - n
    q = s["q"].float().reshape(nb, n, hkv, hq // hkv, D) / math.sqrt(D)
    score = torch.einsum("bnhgd,bkhd->bhgnk", q, k)
    del k
    on, there = _ancestors(_chain(nb, n) if s["parents"] is None else s["parents"], nb, n)
    held = (torch.arange(ctx, device="cuda") < s["ctx_len"][:, None])[:, None, :].expand(nb, n, ctx)
    score.masked_fill_(~torch.cat([held, on], dim=2)[:, None, None], -math.inf)
    score = torch.exp(score - score.amax(dim=-1, keepdim=True).clamp(min=-3e38))
    total = score.sum(dim=-1)
    v = torch.cat([s["v_cache"][table].float().reshape(nb, -1, hkv, D), s["v_new"].float()], dim=1)
    o = torch.einsum("bhgnk,bkhd->bnhgd", score, v) / total.permute(0, 3, 1, 2)[..., None]
    out = s["out"]["o"]
    out.copy_(torch.where(there[:, :, None, None], o.reshape(nb, n, hq, D).to(out.dtype), out))
    return out


def _plain_verify(s):
    c = s["case"]
    nb, n, V = c["B"], c["N"], c["V"]
    b = torch.arange(nb, device="cuda")
    f64 = dict(dtype=torch.float64, device="cuda")

    def target(node):
        x = s["target_logits"][b, node].double() / c["T"]
        e = torch.exp(x - x.amax(dim=1, keepdim=True))
        return e / e.sum(dim=1, keepdim=True)

    node = torch.zeros(nb, dtype=torch.long, device="cuda")
    p, q = target(node), s["draft_q"][b, node].double()
    taken, mass, gone = torch.zeros(nb, **f64), torch.ones(nb, **f64), torch.zeros(nb, **f64)
    length = torch.zeros(nb, dtype=torch.int32, device="cuda")
    path = torch.full((nb, n), -1, dtype=torch.int32, device="cuda")
    path[:, 0] = 0
    for j in range(1, n):  # a verdict on one node is what the next one's depends on
        judged = s["parents"][:, j - 1] == node
        x = s["draft_tokens"][:, j - 1].long()
        px, qx = p[b, x], q[b, x]
        more = mass if c["replacement"] else mass / (1.0 - gone)
        yes = judged & (s["uniforms"][:, j - 1].double() * more * qx < (px - taken * qx).clamp(min=0.0))
        no = judged & ~yes
        taken = torch.where(no, taken + more, torch.where(yes, 0.0, taken))
        gone = torch.where(no, gone + qx, torch.where(yes, 0.0, gone))
        length = length + yes.to(torch.int32)
        path[b, length.long()] = torch.where(yes, j, path[b, length.long()])
        node = torch.where(yes, j, node)
        p, q = target(node), s["draft_q"][b, node].double()
        mass = torch.where(no, (p - taken[:, None] * q).clamp_(min=0.0).sum(dim=1), torch.where(yes, 1.0, mass))
    rest = torch.where((taken > 0)[:, None], (p - taken[:, None] * q).clamp_(min=0.0), p)
    cdf = torch.cumsum(rest, dim=1)
    token = (cdf <= s["uniforms_rs"].double()[:, None] * cdf[:, -1:]).sum(dim=1).to(torch.int32)
    return {"accept_len": length, "path": path, "token": token}


def _plain_append(s):
    c = s["case"]
    nb, n = c["B"], c["N"]
    i = torch.arange(n, device="cuda")
    wanted = i <= s["accept_len"][:, None]
    node = i.expand(nb, n) if s["path"] is None else s["path"].long()
    slot = s["ctx_len"].long()[:, None] + i
    page = s["block_table"].long().gather(1, (slot // c["page"]).clamp(max=s["block_table"].shape[1] - 1))
    seq = torch.arange(nb, device="cuda")[:, None].expand(nb, n)[wanted]
    node, page, slot = node[wanted], page[wanted], (slot % c["page"])[wanted]
    s["k_cache"][:, page, slot] = s["k_new"][:, seq, node]
    s["v_cache"][:, page, slot] = s["v_new"][:, seq, node]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "new_len": s["ctx_len"] + s["accept_len"] + 1}


def run(state):
    if own:
        return _run_own(state)
    return {"adjust": _plain_adjust, "attend": _plain_attend, "verify": _plain_verify, "append": _plain_append}[state["case"]["op"]](state)


# ---- the definitions in 64 bits, sequence by sequence ------------------------------------------


def _up(parents, j):
    """The nodes from j up to the root, or None where there is no node j."""
    way = [j]
    while way[-1] > 0:
        p = parents[way[-1] - 1]
        if p < 0:
            return None
        way.append(p)
    return way


def _exact_adjust(s):
    c = s["case"]
    res = torch.zeros(c["B"], c["N"], c["V"], dtype=torch.float64, device="cuda")
    if c["in_place"]:
        res.copy_(s["logits"])
    parents = [list(range(c["N"] - 1))] * c["B"] if s["parents"] is None else s["parents"].tolist()
    hl, pl = s["history_len"].tolist(), s["prompt_len"].tolist()
    bit = torch.arange(c["V"], device="cuda")
    rows = s["mask_row"].tolist() if s["mask_row"] is not None else None
    for b in range(c["B"]):
        base_all = torch.bincount(s["history"][b, : hl[b]].long(), minlength=c["V"]).double()
        base_out = torch.bincount(s["history"][b, min(pl[b], hl[b]): hl[b]].long(), minlength=c["V"]).double()
        bias = torch.zeros(c["V"], dtype=torch.float64, device="cuda")
        keep = s["bias_tokens"][b] >= 0
        bias[s["bias_tokens"][b][keep].long()] = s["bias_values"][b][keep].double()
        f, pr = s["frequency"][b].double(), s["presence"][b].double()
        for j in range(c["N"]):
            way = _up(parents[b], j)
            if way is None:
                continue
            mine = torch.zeros(c["V"], dtype=torch.float64, device="cuda")
            if len(way) > 1:
                ids = s["draft_tokens"][b][torch.tensor(way[:-1], device="cuda") - 1].long()
                mine.index_put_((ids,), torch.ones(1, dtype=torch.float64, device="cuda"), accumulate=True)
            x = s["logits"][b, j].double()
            if s["repetition"] is not None:
                r = s["repetition"][b].double()
                x = torch.where(base_all + mine > 0, torch.where(x > 0, x / r, x * r), x)
            x = x - f * (base_out + mine) - pr * (base_out + mine > 0).double() + bias
            if rows is not None and rows[b][j] >= 0:
                x[(s["mask"][rows[b][j]][bit // 32] >> (bit % 32)) & 1 == 0] = -math.inf
            res[b, j] = x
    return res


def _exact_attend(s):
    c = s["case"]
    D, hkv, n = c["D"], c["Hkv"], c["N"]
    g = c["Hq"] // hkv
    res = torch.zeros(c["B"], n, c["Hq"], D, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        parents = list(range(n - 1)) if s["parents"] is None else s["parents"][b].tolist()
        L = int(s["ctx_len"][b])
        pages = s["block_table"][b, : -(-L // c["page"])].long()
        ways = [_up(parents, j) for j in range(n)]
        sees = torch.zeros(n, n, dtype=torch.bool)
        for j, way in enumerate(ways):
            if way is not None:
                sees[j, way] = True
        live = [j for j, way in enumerate(ways) if way is not None]
        bar = torch.cat([torch.ones(n, L, dtype=torch.bool), sees], dim=1)[live].cuda()
        for h in range(hkv):
            k = torch.cat([s["k_cache"][pages, :, h].reshape(-1, D)[:L], s["k_new"][b, :, h]]).double()
            v = torch.cat([s["v_cache"][pages, :, h].reshape(-1, D)[:L], s["v_new"][b, :, h]]).double()
            q = s["q"][b, live, h * g:(h + 1) * g].double()
            z = (q @ k.T) * D ** -0.5
            z = z.masked_fill(~bar[:, None], -math.inf)
            w = torch.exp(z - torch.logsumexp(z, dim=-1, keepdim=True))
            res[b, live, h * g:(h + 1) * g] = w @ v
    return res


def _exact_verify(s):
    c = s["case"]
    n, V = c["N"], c["V"]
    par, tok, uni, urs = (s[k].cpu() for k in ("parents", "draft_tokens", "uniforms", "uniforms_rs"))
    lens, toks, paths = [], [], []
    for b in range(c["B"]):
        node, path = 0, [0]
        while True:
            p = torch.softmax(s["target_logits"][b, node].double() / c["T"], dim=0)
            left = s["draft_q"][b, node].double()
            nxt = None
            for j in range(node + 1, n):
                if int(par[b, j - 1]) != node:
                    continue
                x = int(tok[b, j - 1])
                px, qx = float(p[x]), float(left[x])
                if float(uni[b, j - 1]) * qx < px:
                    nxt = j
                    break
                p = (p - left).clamp(min=0)
                p = p / p.sum()
                if not c["replacement"]:
                    left = left.clone()
                    scale = 1.0 - float(left[x])
                    left[x] = 0.0
                    left = left / scale
            if nxt is None:
                break
            node = nxt
            path.append(nxt)
        cdf = torch.cumsum(p, dim=0)
        toks.append(int(torch.searchsorted(cdf, float(urs[b]) * cdf[-1:], right=True)))
        lens.append(len(path) - 1)
        paths.append(path + [-1] * (n - len(path)))
    return {"accept_len": torch.tensor(lens, dtype=torch.int32), "path": torch.tensor(paths, dtype=torch.int32),
            "token": torch.tensor(toks, dtype=torch.int32)}


def exact(case, seed):
    if case["op"] == "append":  # copies: there is nothing to compute
        return None
    return {"adjust": _exact_adjust, "attend": _exact_attend, "verify": _exact_verify}[case["op"]](prepare(case, seed))


# ---- what a pass cannot do without -----------------------------------------------------------


def work(case):
    nb, n, op = case["B"], case["N"], case["op"]
    share = 0.75 if case.get("window") and n > 1 else 1.0  # of the places, those that hold a node
    if op == "adjust":
        V, rows = case["V"], nb * n * share
        banned = case["masked"] * 0.9
        masks = 0 if not case["masked"] else min(64, rows) * V / 8
        if case["in_place"]:  # entries that a penalty or a bias changes, and those that a mask bans
            changed = min(V, 0.35 * case["L"] + 24 + n / 2)
            moved = rows * _size(case) * ((1 - banned) * 2 * changed + banned * V)
        else:
            moved = rows * V * _size(case) * (2.0 - banned)
        return {"bytes": moved + masks + nb * case["L"] * 3.0, "flops": 2.0 * rows * V}
    if op == "attend":
        keys = nb * (case["ctx"] * (9 / 16 if case["ragged"] else 1.0) + n * share)
        return {"bytes": 2.0 * _size(case) * case["D"] * (keys * case["Hkv"] + nb * n * share * case["Hq"]),
                "flops": 4.0 * case["Hq"] * case["D"] * n * share * keys}
    if op == "verify":
        # the walk of the noise model: the chance that a child is taken, children to a node, ways down
        alpha = max(0.3, 1.0 - 0.35 * case["sigma_d"] / math.sqrt(case["T"]))
        wide = max(1.0, min(case["window"] / 2, n * share / 2))
        down = n * share / (1.0 + wide)
        step = 1.0 - (1.0 - alpha) ** wide if n > 1 else 0.0
        visited = 1.0 + sum(step ** i for i in range(1, int(down) + 1))
        refused = min(visited, 1.0 - step ** max(1.0, down) + (visited - 1.0) * (1.0 - alpha)) if n > 1 else 0.0
        return {"bytes": nb * case["V"] * (visited * _size(case) + 4.0 * refused), "flops": 8.0 * nb * case["V"] * visited}
    rows = case["layers"] * nb * (1 + (min(n, 8) - 1) / 2 if case["path"] else 0.75 * n)
    return {"bytes": 4.0 * rows * case["Hkv"] * case["D"] * _size(case), "flops": 0.0}
