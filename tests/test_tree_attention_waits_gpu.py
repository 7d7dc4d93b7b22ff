"""The waits inside the attention kernel, made to run out on purpose (failure detection without a fault): one copy that they depend on is
withheld through the library's test hook (include/dssd_test_hooks.h), with a limit of milliseconds.  The kernel ends by itself, says so per sequence,
and the next ordinary call on the same workspace is right."""
import ctypes

import pytest
import torch

from test_tree_attention_gpu import B, call, make  # noqa: F401

pytestmark = pytest.mark.gpu

NAMES = ("q", "k_new", "v_new", "k_cache", "v_cache", "block_table", "ctx_len")
CYCLES = 20_000_000  # ten milliseconds: a thousand times what an ordinary wait takes


def withhold(B, d, out, ws, seq):  # noqa: F811
    """The hook's call on contiguous tensors."""
    c, p = ctypes, lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())  # noqa: E731
    i64 = lambda t, n: (c.c_int64 * 3)(*t.stride()[:n])  # noqa: E731
    nb, N, Hq, D = d["q"].shape
    f = B.lib.dssd_test_tree_attention_wait_runs_out
    f.restype = c.c_int
    return f(p(d["q"]), i64(d["q"], 3), p(d["k_new"]), p(d["v_new"]), i64(d["k_new"], 3), p(d["k_cache"]), p(d["v_cache"]), i64(d["k_cache"], 3),
             B.DSSD_BF16, p(d["block_table"]), c.c_int64(d["block_table"].shape[1]), d["block_table"].shape[1], d["k_cache"].shape[0], d["k_cache"].shape[1],
             p(d["ctx_len"]), p(d["parents"]), nb, N, Hq, d["k_new"].shape[2], D, c.c_float(D ** -0.5), p(out["o"]), i64(out["o"], 3), p(out["lse"]),
             p(out["flags"]), p(ws), c.c_size_t(ws.numel()), seq, c.c_longlong(CYCLES), None)


def fresh(d, value):
    nb, N, Hq, _ = d["q"].shape
    return {"o": torch.full_like(d["q"], value), "lse": torch.full((nb, N, Hq), value, device="cuda"), "flags": torch.zeros(nb, dtype=torch.int32, device="cuda")}


CASES = [
    # nb, N, Hq, Hkv, D, lens, withheld
    (8, 5, 8, 1, 64, [1000] * 8, 3), (8, 40, 8, 1, 64, [1000] * 8, 3), (6, 3, 8, 2, 128, [700, 0, 90, 5000, 128, 1], 2),
    (5, 30, 16, 2, 128, [129, 300, 2000, 0, 640], 0), (8, 2, 4, 1, 64, [0] * 8, 2),
]


@pytest.mark.parametrize("nb,N,Hq,Hkv,D,lens,seq", CASES)
def test_keys_that_never_arrive(B, nb, N, Hq, Hkv, D, lens, seq):  # noqa: F811
    d = make(61, nb, N, Hq, Hkv, D, 16, lens, torch.bfloat16, chain=True)
    ws = torch.zeros(B.dssd_tree_attention_workspace_bytes(nb, N, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    good = call(B, d, out=fresh(d, 0.0), workspace=ws)
    out = fresh(d, 7.0)
    assert withhold(B, d, out, ws, seq) == B.DSSD_OK
    torch.cuda.synchronize()  # the kernels ended by themselves
    assert int(out["flags"][seq]) == B.CACHE_FLAG_TIMEOUT
    assert (out["flags"] & ~B.CACHE_FLAG_TIMEOUT == 0).all()
    far = [b for b in range(nb) if abs(b - seq) > 3]  # (beyond the pieces that hold the sequence's first tile)
    for b in far:
        assert torch.equal(out["o"][b], good["o"][b]) and torch.equal(out["lse"][b], good["lse"][b]) and int(out["flags"][b]) == 0
    again = call(B, d, out=fresh(d, 3.0), workspace=ws)
    assert all(torch.equal(again[k], good[k]) for k in good)


@pytest.mark.parametrize("nb,N,Hq,Hkv,D,lens,seq", CASES)
def test_a_sequence_without_an_answer_says_so(B, nb, N, Hq, Hkv, D, lens, seq):  # noqa: F811
    """Whatever else the CTAs that gave up had to do: a sequence that does not report a timeout has its answer."""
    d = make(62, nb, N, Hq, Hkv, D, 16, lens, torch.bfloat16, chain=True)
    ws = torch.full((B.dssd_tree_attention_workspace_bytes(nb, N, Hq, Hkv, D),), 1, dtype=torch.uint8, device="cuda")
    good = call(B, d, out=fresh(d, 0.0), workspace=ws)
    ws.fill_(1)  # (as float32 a small positive number: results of nobody)
    out = fresh(d, 7.0)
    assert withhold(B, d, out, ws, seq) == B.DSSD_OK
    torch.cuda.synchronize()
    late = out["flags"] == B.CACHE_FLAG_TIMEOUT
    assert late[seq] and ((out["flags"] == 0) | late).all()
    for b in range(nb):
        row = out["o"][b].float()
        if not late[b]:
            assert torch.equal(out["o"][b], good["o"][b]) and torch.equal(out["lse"][b], good["lse"][b]), b
        else:  # not written, right, or no number: nothing that looks like an answer and is none
            assert ((row == 7.0) | (out["o"][b] == good["o"][b]) | torch.isnan(row)).all(), b
