"""Definitions of the operators of a round on a drafted tree in float64 numpy, sequence by sequence, and inputs for them."""
from __future__ import annotations

import numpy as np
import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}  # half a step, relative


def ways(parents, N):
    """For each node the nodes from it up to the root, or None where there is no node; whether a parent is bad."""
    out, bad = [[0]], False
    for j in range(1, N):
        p = j - 1 if parents is None else int(parents[j - 1])
        if p < 0:
            out.append(None)
        elif p >= j or out[p] is None:
            out.append(None)
            bad = True
        else:
            out.append([j] + out[p])
    return out, bad


def random_parents(rng, B, N, window=4, ragged=True, holes=0.0):
    par = np.full((B, max(0, N - 1)), -1, np.int32)
    for b in range(B):
        n = int(rng.integers((N + 1) // 2, N + 1)) if ragged else N
        for j in range(1, n):
            if rng.random() < holes:
                continue
            up = [p for p in range(max(0, j - window), j) if p == 0 or par[b, p - 1] >= 0]
            par[b, j - 1] = int(rng.choice(up)) if up else -1
    return par


def f64(t):
    return t.detach().double().cpu().numpy()


def adjust(d):
    """Expected logits (float64), the magnitude that roundings are relative to, and the bad-parent flag per sequence."""
    x = f64(d["logits"])
    B, N, V = x.shape
    mag = np.abs(x)
    res = x.copy()
    live = np.zeros((B, N), bool)
    bads = np.zeros(B, bool)

    def get(name, b, default):
        return float(d[name][b]) if d.get(name) is not None else default

    for b in range(B):
        w, bads[b] = ways(None if d.get("parents") is None else d["parents"][b].tolist(), N)
        L = 0 if d.get("history") is None else d["history"].shape[1]
        hl = min(max(int(d["history_len"][b]), 0), L) if L else 0
        pl = min(max(int(d["prompt_len"][b]), 0), hl) if L else 0
        hist = d["history"][b].cpu().numpy() if L else np.zeros(0, np.int64)
        r, pr, fr = get("repetition", b, 1.0), get("presence", b, 0.0), get("frequency", b, 0.0)
        if not (r > 0 and np.isfinite(r)):
            r = 1.0
        for j in range(N):
            if w[j] is None:
                continue
            live[b, j] = True
            n_all, n_out = np.zeros(V), np.zeros(V)
            for i in range(hl):
                v = int(hist[i])
                if 0 <= v < V:
                    n_all[v] += 1
                    n_out[v] += i >= pl
            for k in w[j][:-1]:
                v = int(d["draft_tokens"][b, k - 1])
                if 0 <= v < V:
                    n_all[v] += 1
                    n_out[v] += 1
            y = x[b, j]
            with np.errstate(all="ignore"):
                y = np.where(n_all > 0, np.where(y > 0, y / r, y * r), y)
                mag[b, j] = np.maximum(mag[b, j], np.abs(y)) + abs(fr) * n_out + abs(pr)
                y = np.where(n_out > 0, y - fr * n_out - pr, y)
            if d.get("bias_tokens") is not None:
                bias = {}
                for v, f in zip(d["bias_tokens"][b].tolist(), d["bias_values"][b].tolist()):
                    if 0 <= v < V:
                        bias[v] = f
                for v, f in bias.items():
                    y[v] += f
                    mag[b, j, v] += abs(f)
            if d.get("mask") is not None:
                m = b * N + j if d.get("mask_row") is None else int(d["mask_row"][b, j])
                if 0 <= m < d["mask"].shape[0]:
                    words = d["mask"][m].cpu().numpy().view(np.uint32)
                    ok = (words[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1
                    y = np.where(ok == 1, y, -np.inf)
            res[b, j] = y
    return res, mag, live, bads


def attention(d, scale):
    """o, lse, where there is a node, sum w |v| and the largest scale * sum |q k| (what error bounds are relative to)."""
    q, kn, vn, kc, vc = (f64(d[k]) for k in ("q", "k_new", "v_new", "k_cache", "v_cache"))
    B, N, Hq, D = q.shape
    Hkv, page = kn.shape[2], kc.shape[1]
    table, lens = d["block_table"].cpu().numpy(), d["ctx_len"].cpu().numpy()
    o, wv = np.zeros_like(q), np.zeros_like(q)
    lse, big = np.zeros((B, N, Hq)), np.zeros((B, N, Hq))
    live = np.zeros((B, N), bool)
    for b in range(B):
        L = int(min(max(lens[b], 0), table.shape[1] * page))
        pos = np.arange(L)
        K = np.concatenate([kc[table[b, pos // page], pos % page], kn[b]]) if L else kn[b]
        V = np.concatenate([vc[table[b, pos // page], pos % page], vn[b]]) if L else vn[b]
        w, _ = ways(None if d.get("parents") is None else d["parents"][b].tolist(), N)
        for j in range(N):
            if w[j] is None:
                continue
            live[b, j] = True
            sel = np.concatenate([pos, L + np.array(sorted(w[j]))]).astype(int)
            for h in range(Hq):
                g = h // (Hq // Hkv)
                s = scale * (K[sel, g] @ q[b, j, h])
                m = s.max()
                e = np.exp(s - m)
                lse[b, j, h] = m + np.log(e.sum())
                e /= e.sum()
                o[b, j, h] = e @ V[sel, g]
                wv[b, j, h] = e @ np.abs(V[sel, g])
                big[b, j, h] = scale * (np.abs(K[sel, g]) @ np.abs(q[b, j, h])).max()
    return o, lse, live, wv, big


def verify(d, T, replacement):
    """accept_len, path, token, edge_flags, rs_flags by the definition p <- norm(max(0, p - q)), rejection by rejection."""
    x, q = f64(d["target_logits"]), f64(d["draft_q"]) if d.get("draft_q") is not None else None
    B, N, V = x.shape
    res = {k: np.zeros(B, np.int64) for k in ("accept_len", "token", "edge_flags", "rs_flags")}
    res["path"] = np.full((B, N), -1, np.int64)
    for b in range(B):
        w, bad = ways(None if d.get("parents") is None else d["parents"][b].tolist(), N)
        up = [None] + [w[j][1] if w[j] is not None else None for j in range(1, N)]
        eflags, rflags = (8 if bad else 0), 0
        node, path = 0, [0]
        while True:
            l = x[b, node] / T
            with np.errstate(all="ignore"):
                top = l.max() if not np.isnan(l).any() else np.nan
                p = np.exp(l - top)
                p = p / p.sum()
            alive = np.isfinite(top)
            if not alive:
                eflags |= 2
            p0, nxt, child = p, None, False
            left = q[b, node].copy() if q is not None and N > 1 else None
            for j in range(node + 1, N):
                if up[j] != node:
                    continue
                child = True
                t = int(d["draft_tokens"][b, j - 1])
                u = float(d["uniforms"][b, j - 1])
                ok = 0 <= t < V
                if not ok:
                    eflags |= 1
                elif alive and u < 1 and (p[t] > 0 if left[t] <= 0 else u * left[t] < p[t]):
                    nxt = j
                    break
                with np.errstate(all="ignore"):
                    r = p - left
                    r = np.where(r > 0, r, 0)
                    p = r / r.sum() if r.sum() > 0 else r
                    if ok and not replacement and left[t] > 0:
                        left[t] = 0
                        left = left / left.sum() if left.sum() > 0 else left
            if nxt is None:
                break
            node = nxt
            path.append(nxt)
        if not child:
            rflags |= 1
        if child and not p.sum() > 0 and alive:
            rflags |= 2
            p = p0
        if not alive:  # after a rejection the fallback finds no mass either
            rflags |= 4 | (2 if child else 0)
            token = -1
        else:
            cdf = np.cumsum(p)
            over = np.nonzero(cdf > float(d["uniforms_rs"][b]) * cdf[-1])[0]
            token = int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1])
        res["accept_len"][b], res["token"][b] = len(path) - 1, token
        res["path"][b, : len(path)] = path
        res["edge_flags"][b], res["rs_flags"][b] = eflags, rflags
    return res


def verify_inputs(rng, B, N, V, dtype, T=1.0, sigma=0.7, replacement=True, window=4, ragged=True, parents="tree"):
    """Target logits, draft rows, tokens drawn from them with or without replacement, uniforms; on the GPU."""
    x = torch.from_numpy((rng.normal(0, 2.0, (B, N, V)) - 1.1 * np.log1p(rng.permutation(V)))).to(dtype)
    z = (x.double().numpy() + rng.normal(0, sigma, (B, N, V))) / T
    q = np.exp(z - z.max(axis=2, keepdims=True))
    q = (q / q.sum(axis=2, keepdims=True)).astype(np.float32)
    par = None if parents is None else random_parents(rng, B, N, window, ragged)
    tok = np.zeros((B, max(0, N - 1)), np.int32)
    for b in range(B):
        gone = {}
        for j in range(1, N):
            p = j - 1 if par is None else max(0, int(par[b, j - 1]))
            w = q[b, p].astype(np.float64).copy()
            if not replacement:
                w[gone.get(p, [])] = 0
                if w.sum() <= 0:
                    w = q[b, p].astype(np.float64).copy()
            t = int(np.searchsorted(np.cumsum(w), rng.random() * w.sum(), side="right"))
            tok[b, j - 1] = min(t, V - 1)
            gone.setdefault(p, []).append(tok[b, j - 1])
    u = (rng.integers(0, 1 << 24, (B, max(0, N - 1))) * 2.0 ** -24).astype(np.float32)
    ur = (rng.integers(0, 1 << 24, B) * 2.0 ** -24).astype(np.float32)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return {"target_logits": x.cuda(), "draft_q": up(q), "draft_tokens": up(tok), "parents": None if par is None else up(par),
            "uniforms": up(u), "uniforms_rs": up(ur)}
