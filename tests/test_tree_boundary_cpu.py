"""What the entry points of a round on a drafted tree refuse on the host, before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2507_12000_b200 import build

    build.build()
    from paper_2507_12000_b200 import binding

    return binding


P = 0x10000  # an address that is never looked at


def i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def adjust(B, /, **kw):
    a = dict(logits=P, dtype=0, row_stride=100, B=2, N=3, V=100, draft_tokens=P, parents=None, history=P, history_stride=9, L=9, prompt_len=P,
             history_len=P, repetition=None, presence=None, frequency=None, bias_tokens=P, bias_values=P, K=4, mask=P, mask_rows=2, mask_row=P,
             out=2 * P, out_stride=100, flags=None, workspace=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return B.lib.dssd_adjust_logits(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), 1), (dict(out=None), 1), (dict(B=0), 1), (dict(N=0), 1), (dict(V=0), 1), (dict(row_stride=99), 1), (dict(out_stride=99), 1),
    (dict(out=P, out_stride=101), 1), (dict(draft_tokens=None), 1), (dict(L=-1), 1), (dict(history=None), 1), (dict(history_len=None), 1),
    (dict(prompt_len=None), 1), (dict(history_stride=8), 1), (dict(bias_tokens=None), 1), (dict(bias_values=None), 1), (dict(K=-1), 1),
    (dict(mask=None), 1), (dict(mask_row=None), 1), (dict(mask_rows=-1), 1), (dict(logits=P + 2), 1), (dict(dtype=2), 2), (dict(dtype=9), 2),
    (dict(N=129), 2), (dict(K=65536), 2), (dict(L=1 << 29, history_stride=1 << 29), 2), (dict(V=(1 << 30) + 1, row_stride=1 << 31, out_stride=1 << 31), 2),
    (dict(V=(1 << 24) + 1, row_stride=1 << 31, out_stride=1 << 31), 2), (dict(workspace=None), 3), (dict(workspace=P + 8), 3), (dict(bytes=0), 3),
])
def test_adjust_refuses(B, kw, status):
    assert adjust(B, **kw) == status


def attend(B, /, **kw):
    a = dict(q=P, q_strides=i64(1024, 512, 128), k_new=P, v_new=P, new_strides=i64(1024, 256, 128), k_cache=P, v_cache=P,
             cache_strides=i64(4096, 256, 128), dtype=1, block_table=P, table_stride=8, max_pages=8, num_pages=20, page_size=16, ctx_len=P, parents=None,
             B=2, N=2, Hq=4, Hkv=2, D=128, scale=0.1, o=P, o_strides=i64(1024, 512, 128), lse=None, flags=None, workspace=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return B.lib.dssd_tree_attention(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(k_new=None), 1), (dict(v_new=None), 1), (dict(o=None), 1), (dict(ctx_len=None), 1), (dict(block_table=None), 1),
    (dict(k_cache=None), 1), (dict(q_strides=None), 1), (dict(B=0), 1), (dict(N=0), 1), (dict(Hq=3), 1), (dict(Hkv=0), 1), (dict(D=0), 1),
    (dict(page_size=0), 1), (dict(table_stride=7), 1), (dict(num_pages=-1), 1), (dict(max_pages=-1), 1), (dict(scale=0.0), 1),
    (dict(scale=float("nan")), 1), (dict(q=P + 8), 1), (dict(v_cache=P + 2), 1), (dict(o=P + 4), 1), (dict(q_strides=i64(1024, -512, 128)), 1),
    (dict(dtype=0), 2), (dict(N=129), 2), (dict(D=12), 2), (dict(D=136), 2), (dict(Hq=258, Hkv=2), 2), (dict(new_strides=i64(1024, 256, 130)), 2),
    (dict(q_strides=i64(0, 512, 128)), 2), (dict(new_strides=i64(1024, 256, 0)), 2), (dict(cache_strides=i64(0, 256, 128)), 2),
    (dict(max_pages=1 << 20, table_stride=1 << 20, page_size=1 << 12), 2), (dict(workspace=None), 3), (dict(workspace=P + 16), 3), (dict(bytes=0), 3),
])
def test_attention_refuses(B, kw, status):
    assert attend(B, **kw) == status


def verify(B, /, **kw):
    a = dict(logits=P, dtype=0, row_stride=100, draft_q=P, draft_tokens=P, parents=None, uniforms=P, uniforms_rs=P, T=1.0, replacement=1, B=2, N=3, V=100,
             accept_len=P, path=P, token=P, edge_flags=None, rs_flags=None, workspace=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return B.lib.dssd_tree_verify(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), 1), (dict(draft_q=None), 1), (dict(draft_tokens=None), 1), (dict(uniforms=None), 1), (dict(uniforms_rs=None), 1),
    (dict(accept_len=None), 1), (dict(path=None), 1), (dict(token=None), 1), (dict(T=0.0), 1), (dict(T=float("inf")), 1), (dict(row_stride=99), 1),
    (dict(B=0), 1), (dict(N=0), 1), (dict(V=0), 1), (dict(logits=P + 2), 1), (dict(draft_q=P + 1), 1), (dict(dtype=2), 2), (dict(N=129), 2), (dict(T=2e30), 2),
    (dict(workspace=None), 3), (dict(workspace=P + 8), 3), (dict(bytes=0), 3),
])
def test_verify_refuses(B, kw, status):
    assert verify(B, **kw) == status


def append(B, /, **kw):
    a = dict(k_new=P, v_new=P, new_strides=i64(0, 1024, 256, 128), k_cache=P, v_cache=P, cache_strides=i64(0, 4096, 256, 128), dtype=1, block_table=P,
             table_stride=8, max_pages=8, num_pages=20, page_size=16, ctx_len=P, accept_len=P, path=None, layers=1, B=2, N=4, Hkv=2, D=128,
             new_len=2 * P, flags=None, stream=None)
    a.update(kw)
    return B.lib.dssd_cache_append(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(k_new=None), 1), (dict(v_cache=None), 1), (dict(ctx_len=None), 1), (dict(accept_len=None), 1), (dict(block_table=None), 1),
    (dict(new_len=P), 1), (dict(layers=0), 1), (dict(N=0), 1), (dict(page_size=0), 1), (dict(k_new=P + 1), 1), (dict(new_strides=i64(0, -1, 256, 128)), 1),
    (dict(dtype=0), 2), (dict(layers=40000, B=40000, N=4), 2), (dict(max_pages=1 << 20, table_stride=1 << 20, page_size=1 << 12), 2),
])
def test_append_refuses(B, kw, status):
    assert append(B, **kw) == status


def test_workspace_sizes_never_decrease(B):
    f, g = B.dssd_tree_attention_workspace_bytes, B.dssd_tree_verify_workspace_bytes
    assert f(0, 1, 8, 8, 64) == f(1, 129, 8, 8, 64) == f(1, 1, 3, 2, 64) == f(1, 1, 8, 8, 12) == g(1, 129, 10) == g(1, 1, 0) == 0
    sizes = [f(b, n, 8 * h, h, d) for b in (1, 40) for n in (1, 33) for h in (1, 8) for d in (8, 128)]
    assert all(s > 0 and s % 256 == 0 for s in sizes)
    for a in ((1, 1, 8, 8, 64), (3, 17, 32, 8, 96)):
        for k in range(5):
            more = list(a)
            more[k] *= 2 if k != 3 else 1
            if k == 4:
                more[k] = 128
            assert f(*more) >= f(*a)
    h = B.dssd_adjust_logits_workspace_bytes
    assert h(0, 1, 10, 0, 0) == h(1, 129, 10, 0, 0) == h(1, 1, (1 << 24) + 1, 0, 0) == h(1, 1, 10, -1, 0) == h(1, 1, 10, 0, 65536) == 0
    for a in ((1, 1, 1, 0, 0), (3, 17, 50272, 600, 32)):
        for k in range(5):
            more = list(a)
            more[k] = 2 * more[k] + 1
            assert h(*more) >= h(*a) > 0
    assert g(1, 2, 100) <= g(2, 2, 100) <= g(2, 128, 100) <= g(2, 128, 200000)


def test_the_front_end_refuses(B):
    z = torch.zeros
    with pytest.raises(AssertionError):  # not CUDA tensors
        B.dssd_adjust_logits(z(1, 2, 8))
    with pytest.raises(AssertionError):
        B.dssd_tree_verify(z(1, 1, 8), None, None, None, None, z(1), 1.0, out={}, workspace=z(256, dtype=torch.uint8))
    h = z(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        B.dssd_tree_attention(h, h, h, h, h, z(1, 1, dtype=torch.int32), z(1, dtype=torch.int32), workspace=z(256, dtype=torch.uint8))
    k = z(1, 1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        B.dssd_cache_append(k, k, k, k, z(1, 1, dtype=torch.int32), z(1, dtype=torch.int32), z(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        B._marshal.tree_verify(h)
