"""A round on a drafted tree: what happens between the target model's forward pass and the next draft.

The device drafts N - 1 candidate tokens that form a tree under the last committed token (the root); the target model
scores all nodes in one forward pass, its attention layers through `binding.dssd_tree_attention`.  `verify_round_tree` takes
the logits of that pass and finishes the round: penalties, biases and masks on every node's row, the verdict (Algorithm 1's
test and residual, where a position has several candidates), and the accepted path's keys and values into the
cache of all layers.  Nothing waits for the GPU, so that a whole round can be captured in a CUDA graph.

Every step of the method, from the logits to the verdict and the cache, runs in the library's kernels; what is put together here with torch's own is the list of
emitted tokens, for the caller's convenience (`emitted_tokens`, about ten small kernels).
"""
from __future__ import annotations

from typing import Dict, Optional

import torch


def verify_round_tree(target_logits: torch.Tensor, draft_q: Optional[torch.Tensor], draft_tokens: Optional[torch.Tensor],
                      parents: Optional[torch.Tensor], uniforms: Optional[torch.Tensor], uniforms_rs: torch.Tensor,
                      temperature: float, *, replacement: bool = True, adjust: Optional[Dict[str, torch.Tensor]] = None,
                      cache: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> Dict[str, torch.Tensor]:
    """One round.  target_logits [B, N, V] (adjusted in place if `adjust` is given), draft_q, draft_tokens, parents,
    uniforms, uniforms_rs, replacement as for `dssd_tree_verify`.  stream: as the calls take it (None, a torch stream, a handle); everything
    runs there.

    adjust: the arguments of `dssd_adjust_logits` by name (history, prompt_len, history_len, repetition, presence, frequency,
            bias_tokens, bias_values, mask, mask_row), those that are wanted.
    cache:  k_new, v_new [layers, B, N, Hkv, D] of this pass and k_cache, v_cache, block_table, ctx_len; the path is appended.

    Returns what `dssd_tree_verify` does, `tokens` [B, N] (the accepted drafted tokens and the drawn one in order, then -1), and with a cache
    `new_len` and `cache_flags`, with adjustments `adjust_flags`."""
    from . import binding as B

    dev = target_logits.device
    stream = B.as_stream(stream, dev)  # (what is no stream is refused before anything is written)
    result: Dict[str, torch.Tensor] = {}
    if adjust is not None:
        out = B._made(stream, dev, lambda: {"flags": torch.empty(target_logits.shape[0], dtype=torch.int32, device=dev)})
        out["logits"] = target_logits
        B.dssd_adjust_logits(target_logits, draft_tokens=draft_tokens, parents=parents, out=out, stream=stream, **adjust)
        result["adjust_flags"] = out["flags"]
    result.update(B.dssd_tree_verify(target_logits, draft_q, draft_tokens, parents, uniforms, uniforms_rs, temperature,
                                     replacement=replacement, stream=stream))
    if cache is not None:
        a = B.dssd_cache_append(cache["k_new"], cache["v_new"], cache["k_cache"], cache["v_cache"], cache["block_table"],
                                cache["ctx_len"], result["accept_len"], path=result["path"], stream=stream)
        result["new_len"], result["cache_flags"] = a["new_len"], a["flags"]
    result["tokens"] = emitted_tokens(result["path"], draft_tokens, result["accept_len"], result["token"], stream)
    return result


def emitted_tokens(path: torch.Tensor, draft_tokens: Optional[torch.Tensor], accept_len: torch.Tensor, token: torch.Tensor,
                   stream=None) -> torch.Tensor:
    """[B, N]: the tokens of the accepted nodes, then the drawn token, then -1."""
    if stream is not None:
        from . import binding as B

        return B._made(stream, path.device, lambda: emitted_tokens(path, draft_tokens, accept_len, token))
    n = path.shape[1]
    at = torch.arange(n, device=path.device)
    last = token[:, None].expand(-1, n)
    if n > 1:
        ahead = torch.cat([path[:, 1:], path[:, :1]], dim=1).long()  # node of the i-th emitted token
        drafted = draft_tokens.gather(1, (ahead - 1).clamp(min=0))
        last = torch.where(at < accept_len[:, None], drafted, last)
    return torch.where(at <= accept_len[:, None], last, torch.full_like(path, -1))
