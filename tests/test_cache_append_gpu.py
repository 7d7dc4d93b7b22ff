"""dssd_cache_append: the rows that should move have moved, nothing else has changed."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2507_12000_b200 import binding

    return binding


def expected(kc, vc, kn, vn, table, ctx, acc, path, page):
    kc, vc = kc.clone(), vc.clone()
    nb, N = kn.shape[1], kn.shape[2]
    flags = np.zeros(nb, np.int64)
    new = np.zeros(nb, np.int64)
    for b in range(nb):
        n = max(0, min(int(acc[b]), N - 1) + 1)
        if int(acc[b]) >= N:
            flags[b] |= 4
        new[b] = int(ctx[b]) + n
        for i in range(n):
            node = i if path is None else int(path[b, i])
            pos = int(ctx[b]) + i
            ok = 0 <= node < N
            flags[b] |= 0 if ok else 4
            if int(ctx[b]) < 0 or pos // page >= table.shape[1]:
                flags[b] |= 2
                continue
            pg = int(table[b, pos // page])
            if not 0 <= pg < kc.shape[1]:
                flags[b] |= 1
                continue
            if ok:
                kc[:, pg, pos % page] = kn[:, b, node]
                vc[:, pg, pos % page] = vn[:, b, node]
    return kc, vc, new, flags


def make(rng, L, nb, N, H, D, page, dtype, spare=2):
    per = -(-(40 + N) // page)
    total = nb * per + spare
    t = lambda *s: torch.randn(*s, device="cuda").to(dtype)  # noqa: E731
    table = torch.from_numpy(rng.permutation(total)[: nb * per].reshape(nb, per).astype(np.int32)).cuda()
    ctx = torch.from_numpy(rng.integers(0, 40, nb).astype(np.int32)).cuda()
    acc = torch.from_numpy(rng.integers(-1, N, nb).astype(np.int32)).cuda()
    return t(L, nb, N, H, D), t(L, nb, N, H, D), t(L, total, page, H, D), t(L, total, page, H, D), table, ctx, acc


def check(B, kn, vn, kc, vc, table, ctx, acc, path, **kw):
    ek, ev, new, flags = expected(kc, vc, kn, vn, table, ctx, acc, path, kc.shape[2])
    r = B.dssd_cache_append(kn, vn, kc, vc, table, ctx, acc, path=path, **kw)
    torch.cuda.synchronize()
    assert torch.equal(kc.view(torch.int16), ek.view(torch.int16)) and torch.equal(vc.view(torch.int16), ev.view(torch.int16))
    assert (r["new_len"].cpu().numpy() == new).all() and (r["flags"].cpu().numpy() == flags).all()


@pytest.mark.parametrize("L,nb,N,H,D,page,dtype", [
    (1, 1, 1, 1, 8, 1, torch.float16), (3, 5, 16, 4, 128, 16, torch.bfloat16), (9, 2, 7, 3, 64, 5, torch.float16), (4, 3, 8, 1, 7, 8, torch.bfloat16),
    (1, 4, 300, 2, 96, 48, torch.bfloat16), (33, 1, 2, 8, 128, 256, torch.bfloat16), (2, 70, 9, 2, 20, 16, torch.float16),
])
@pytest.mark.parametrize("with_path", [False, True])
def test_rows_move(B, L, nb, N, H, D, page, dtype, with_path):
    rng = np.random.default_rng(L * 100 + N)
    kn, vn, kc, vc, table, ctx, acc = make(rng, L, nb, N, H, D, page, dtype)
    path = None
    if with_path:
        p = np.full((nb, N), -1, np.int32)
        for b in range(nb):
            n = int(acc[b]) + 1
            p[b, :n] = np.sort(rng.choice(N, n, replace=False))
        path = torch.from_numpy(p).cuda()
    check(B, kn, vn, kc, vc, table, ctx, acc, path)


def test_views_of_one_buffer(B):
    """Keys and values of one projection, caches of one allocation with the heads before the positions."""
    rng = np.random.default_rng(1)
    L, nb, N, H, D, page = 2, 3, 5, 2, 32, 4
    _, _, _, _, table, ctx, acc = make(rng, L, nb, N, H, D, page, torch.bfloat16)
    qkv = torch.randn(L, nb, N, 3 * H, D, device="cuda").bfloat16()
    both = torch.randn(2, L, int(table.max()) + 3, H, page, D, device="cuda").bfloat16()
    kc, vc = both[0].transpose(2, 3), both[1].transpose(2, 3)
    check(B, qkv[:, :, :, H:2 * H], qkv[:, :, :, 2 * H:], kc, vc, table, ctx, acc, None)


def test_bad_pages_nodes_and_lengths_are_skipped(B):
    rng = np.random.default_rng(2)
    kn, vn, kc, vc, table, ctx, acc = make(rng, 2, 6, 6, 2, 16, 4, torch.float16)
    acc[:] = torch.tensor([5, 3, 6, 2, 5, 1], dtype=torch.int32)
    ctx[:] = torch.tensor([3, 0, 1, 4 * table.shape[1] - 1, -2, 5], dtype=torch.int32)
    table[0, 1], table[1, 0] = kc.shape[1], -1
    path = torch.arange(6, dtype=torch.int32, device="cuda").expand(6, 6).contiguous()
    path[5, 1] = 6
    check(B, kn, vn, kc, vc, table, ctx, acc, path)


def test_places_beyond_32_bits(B):
    """A cache of more than 2^32 bytes and 2^31 elements: the last page."""
    pages = (1 << 31) // (16 * 2 * 128) + 2
    kc = torch.zeros(1, pages, 16, 2, 128, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    kn = torch.randn(1, 1, 2, 2, 128, device="cuda").bfloat16()
    vn = torch.randn(1, 1, 2, 2, 128, device="cuda").bfloat16()
    table = torch.tensor([[0, pages - 1]], dtype=torch.int32, device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    B.dssd_cache_append(kn, vn, kc, vc, table, 15 * one, one)
    torch.cuda.synchronize()
    assert torch.equal(kc[0, 0, 15], kn[0, 0, 0]) and torch.equal(kc[0, -1, 0], kn[0, 0, 1]) and torch.equal(vc[0, -1, 0], vn[0, 0, 1])
    assert int((kc != 0).any(dim=-1).any(dim=-1).sum()) == 2


def test_in_a_graph_on_another_stream(B):
    rng = np.random.default_rng(3)
    kn, vn, kc, vc, table, ctx, acc = make(rng, 2, 3, 4, 2, 16, 4, torch.float16)
    out = {"new_len": torch.zeros(3, dtype=torch.int32, device="cuda"), "flags": torch.zeros(3, dtype=torch.int32, device="cuda")}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.dssd_cache_append(kn, vn, kc, vc, table, ctx, acc, out=out)
    kn.add_(1)
    ek, ev, new, _ = expected(kc, vc, kn, vn, table, ctx, acc, None, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g.replay()
    s.synchronize()
    assert torch.equal(kc, ek) and torch.equal(vc, ev) and (out["new_len"].cpu().numpy() == new).all()
