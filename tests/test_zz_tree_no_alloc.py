"""The calls of a round on a drafted tree allocate nothing on the device when they are given their outputs and workspace.  Collected last, like the test of
the entry point that cannot allocate."""
import numpy as np
import pytest
import torch

import tree_ref as R
from test_tree_attention_gpu import make

pytestmark = pytest.mark.gpu


def test_no_call_takes_device_memory():
    from paper_2507_12000_b200 import binding as B

    v = R.verify_inputs(np.random.default_rng(3), 4, 9, 5000, torch.bfloat16)
    d = make(3, 4, 9, 8, 2, 64, 16, [3000, 40, 0, 700], torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    hist, one = i32(4, 20000), torch.ones(4, dtype=torch.int32, device="cuda")
    space = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    adjusted = {"logits": torch.zeros_like(v["target_logits"]), "flags": i32(4)}
    in_place = {"logits": adjusted["logits"], "flags": i32(4)}
    verdict = {**{k: i32(4) for k in ("accept_len", "token", "edge_flags", "rs_flags")}, "path": i32(4, 9)}
    attended = {"o": torch.zeros_like(d["q"]), "lse": torch.zeros(4, 9, 8, device="cuda"), "flags": i32(4)}
    appended = {"new_len": i32(4), "flags": i32(4)}
    ws_adjust, ws_verify = space(B.dssd_adjust_logits_workspace_bytes(4, 9, 5000, 20000, 0)), space(B.dssd_tree_verify_workspace_bytes(4, 9, 5000))
    ws_attend = space(B.dssd_tree_attention_workspace_bytes(4, 9, 8, 2, 64))
    names = ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")
    length, per = one * 20000, torch.ones(4, device="cuda")
    layer = {k: d[k][None] for k in ("k_new", "v_new", "k_cache", "v_cache")}

    def round_():
        B.dssd_tree_attention(*[d[k] for k in names], parents=d["parents"], out=attended, workspace=ws_attend)
        for x, out in ((v["target_logits"], adjusted), (adjusted["logits"], in_place)):
            B.dssd_adjust_logits(x, hist, one, length, draft_tokens=v["draft_tokens"], parents=v["parents"], frequency=per, out=out, workspace=ws_adjust)
        for replacement in (True, False):
            B.dssd_tree_verify(adjusted["logits"], v["draft_q"], v["draft_tokens"], v["parents"], v["uniforms"], v["uniforms_rs"], 1.0, replacement=replacement,
                               out=verdict, workspace=ws_verify)
        B.dssd_cache_append(*layer.values(), d["block_table"], d["ctx_len"], one * 0 - 1, out=appended)

    round_()  # (kernels are loaded on their first launch)
    torch.cuda.synchronize()
    state = torch.cuda.mem_get_info()[0], torch.cuda.memory_reserved()
    for _ in range(3):
        round_()
    torch.cuda.synchronize()
    assert (torch.cuda.mem_get_info()[0], torch.cuda.memory_reserved()) == state
