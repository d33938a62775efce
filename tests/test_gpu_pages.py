"""The calls on pages on the GPU against the plain reference, on caches of every type."""
import numpy as np
import pytest

from tests import pages_util as P

pytestmark = pytest.mark.gpu
PAGE = 64


def _cache(rng, pages, bits8, heads=4, page=PAGE, block=32):
    """What a page holds: index keys, K, V, and the 8-bit cache's scales and block keys."""
    import torch
    n = page // block
    shapes = [((page, 4, 64), 2)] + [((page, heads, 128), 1 if bits8 else 2)] * 2
    if bits8:
        shapes += [((n, heads), 4)] * 2 + [((n, 256), 2)]
    kinds = {1: torch.uint8, 2: torch.int16, 4: torch.int32}
    return [torch.from_numpy(rng.integers(0, 256, (pages, int(np.prod(s)) * b), dtype=np.uint8)).cuda()
            .view(kinds[b]).reshape((pages, *s)) for s, b in shapes]


def _moved(before, moves):
    import torch
    out = [b.clone() for b in before]
    if moves:
        a, z = (torch.tensor(m, device="cuda") for m in zip(*moves))
        for o, b in zip(out, before):
            o[z] = b[a]
    return out


def _same(ts, want):
    import torch
    return all(torch.equal(a, b) for a, b in zip(ts, want))


def _dev(*xs):
    import torch
    return [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in xs]


def _shape(batch, cols, n_q=1, page=PAGE):
    from paper_2606_06467_amd import binding as B
    return B.make_shape(batch, n_q, cols * page, 1, page_size=page, max_pages=cols)


@pytest.mark.parametrize("batch,cols,bad", [(1, 1, 0), (8, 9, 0), (64, 513, 0), (2000, 20, 0), (16384, 3, 0), (11, 70, 0.1)])
def test_fork(batch, cols, bad):
    from paper_2606_06467_amd import binding as B
    rng = np.random.default_rng(batch + cols)
    pages = batch * cols // 2 + 9
    table, refs = P.state(rng, batch, cols, pages, bad=bad, pinned=3)
    lens = rng.integers(0, cols * PAGE, batch).astype(np.int32)
    parent = np.where(rng.random(batch) < 0.3, np.arange(batch), rng.integers(-1, batch, batch)).astype(np.int32)
    if bad:
        parent[:2] = [batch, -2]
    want = P.fork(parent, table, lens, refs)
    t, l, r, p = _dev(table, lens, refs, parent)
    B.clsa_get_device_error()
    B.clsa_pages_fork(_shape(batch, cols), p, t, l, r)
    for x, w in zip((t, l, r), want):
        assert np.array_equal(x.cpu().numpy(), w)
    assert B.clsa_get_device_error() == (B.CLSA_DEVERR_PAGES if want[3] else 0)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("batch,cols,n_q,spare,page", [(1, 4, 1, 9, 64), (6, 9, 1, 99, 64), (40, 30, 300, 1500, 16),
                                                       (3000, 3, 1, 200, 16), (5, 6, 900, 40, 128), (12, 9, 4, 3, 64), (700, 4, 1, 900, 16),
                                                       (300, 9, 40, 5000, 16)])
def test_reserve(bits8, batch, cols, n_q, spare, page):
    from paper_2606_06467_amd import binding as B
    rng = np.random.default_rng(batch * cols + n_q)
    heads = 1 if batch >= 300 else 4
    pages = batch * cols // 2 + spare
    table, refs = P.state(rng, batch, cols, pages, shared=0.7, pinned=2)
    start = rng.integers(0, cols * page + 1, batch).astype(np.int32)
    count = np.minimum(rng.integers(0, n_q + 1, batch), cols * page - start).astype(np.int32)
    t, r, copies, missing = P.reserve(start, count, table, refs, n_q, page, cols * page)
    cache = _cache(rng, pages, bits8, heads, page, 16)
    want = _moved(cache, copies)
    T, R, S, N = _dev(table, refs, start, count)
    M, = _dev(np.full(1, 5, np.int32))
    sh = _shape(batch, cols, n_q, page)
    ws = B.workspace(sh, B.CLSA_OP_PAGES_RESERVE)
    ws.fill_(0xFF)
    B.clsa_get_device_error()
    B.clsa_pages_reserve(sh, cache, S, N, T, R, M, ws)
    assert np.array_equal(T.cpu().numpy(), t) and np.array_equal(R.cpu().numpy(), r) and int(M[0]) == missing
    assert _same(cache, want)
    assert B.clsa_get_device_error() == (B.CLSA_DEVERR_PAGES if missing else 0)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("batch,cols,pages,pinned", [(1, 1, 1, 0), (7, 9, 60, 0), (30, 40, 2000, 12), (50, 3, 5000, 0),
                                                     (9, 6, 54, 54), (40, 300, 9001, 4), (700, 64, 4000, 0)])
def test_compact(bits8, batch, cols, pages, pinned):
    from paper_2606_06467_amd import binding as B
    rng = np.random.default_rng(pages)
    table, refs = P.state(rng, batch, cols, pages, shared=0.6, pinned=pinned)
    t, r, moves, bound = P.compact(table, refs)
    cache = _cache(rng, pages, bits8, 1, 16, 16)
    want = _moved(cache, moves)
    T, R = _dev(table, refs)
    M, = _dev(np.full(1, 5, np.int32))
    sh = _shape(batch, cols, page=16)
    ws = B.workspace(sh, B.CLSA_OP_PAGES_COMPACT, pages)
    ws.fill_(0xFF)
    B.clsa_pages_compact(sh, cache, T, R, M, ws)
    assert np.array_equal(T.cpu().numpy(), t) and np.array_equal(R.cpu().numpy(), r) and int(M[0]) == bound
    assert _same(cache, want)
    # nothing is left to move
    B.clsa_pages_compact(sh, cache, T, R, M, ws)
    assert np.array_equal(T.cpu().numpy(), t) and np.array_equal(R.cpu().numpy(), r) and _same(cache, want)


def test_compact_past_the_caches():
    """Enough pages that the copies are streamed."""
    from paper_2606_06467_amd import binding as B
    rng = np.random.default_rng(1)
    pages, batch, cols = 3000, 20, 75
    table = np.full((batch, cols), -1, np.int32)
    table[:] = rng.permutation(pages)[:batch * cols].reshape(batch, cols)
    refs = P.holders(table, pages)
    t, r, moves, bound = P.compact(table, refs)
    cache = _cache(rng, pages, False)
    assert len(moves) * sum(c[0].nbytes for c in cache) > 64 << 20
    want = _moved(cache, moves)
    T, R = _dev(table, refs)
    M, = _dev(np.zeros(1, np.int32))
    sh = _shape(batch, cols)
    B.clsa_pages_compact(sh, cache, T, R, M, B.workspace(sh, B.CLSA_OP_PAGES_COMPACT, pages))
    assert np.array_equal(T.cpu().numpy(), t) and np.array_equal(R.cpu().numpy(), r) and int(M[0]) == bound
    assert _same(cache, want)


def test_copy():
    import torch
    from paper_2606_06467_amd import binding as B
    rng = np.random.default_rng(4)
    cache = _cache(rng, 300, True)
    cache.append(torch.arange(300 * 5, dtype=torch.int32, device="cuda").view(300, 5))  # 20 bytes a page
    perm = rng.permutation(300)
    src, dst = perm[:120].astype(np.int32), perm[150:270].astype(np.int32)
    src[7] = -1
    want = _moved(cache, [(int(a), int(z)) for a, z in zip(src, dst) if a >= 0])
    B.clsa_pages_copy(cache, *_dev(src, dst))
    assert _same(cache, want)
    B.clsa_pages_copy(cache, *_dev(src[:0], dst[:0]))
    with pytest.raises(ValueError):
        B.clsa_pages_copy(cache, *_dev(src[:3], dst[:2]))


def test_copy_of_offsets_past_32_bits():
    import torch
    from paper_2606_06467_amd import binding as B
    pages, width = 70000, 1 << 16
    x = torch.zeros((pages, width), dtype=torch.uint8, device="cuda")  # 4.6 GB
    x[69999], x[2] = 7, 9
    src, dst = _dev(np.array([69999, 2], np.int32), np.array([1, 69998], np.int32))
    B.clsa_pages_copy([x], src, dst)
    assert bool((x[1] == 7).all()) and bool((x[69998] == 9).all()) and bool((x[69999] == 7).all())
    assert int(x.view(pages, -1)[:, 0].ne(0).sum()) == 4


def test_captured_twice_with_one_workspace_each():
    """Two captured steps of fork and reserve, replayed in turn, against the same steps run eagerly."""
    import torch
    from paper_2606_06467_amd import binding as B
    rng = np.random.default_rng(9)
    batch, cols, pages = 12, 10, 400
    table, refs = P.state(rng, batch, cols, pages, shared=0.0)
    lens = ((table >= 0).sum(1) * PAGE - rng.integers(0, 40, batch)).clip(0).astype(np.int32)
    cache0 = _cache(rng, pages, False)
    parents = [rng.integers(0, batch, batch).astype(np.int32), rng.integers(-1, batch, batch).astype(np.int32)]
    count = np.where(lens + 30 <= cols * PAGE, 30, 0).astype(np.int32)
    sh = _shape(batch, cols, 32)

    def fresh():
        T, L, R = _dev(table, lens, refs)
        return T, L, R, [c.clone() for c in cache0], torch.zeros(1, dtype=torch.int32, device="cuda")

    N, *PP = _dev(count, *parents)
    zero = torch.zeros_like(N)

    def step(i, st, ws):
        T, L, R, cache, M = st
        B.clsa_pages_fork(sh, PP[i], T, L, R)
        B.clsa_pages_reserve(sh, cache, L, torch.where(L + 32 <= cols * PAGE, N, zero), T, R, M, ws)

    eager = fresh()
    for i in (0, 1, 0, 0, 1):
        step(i, eager, B.workspace(sh, B.CLSA_OP_PAGES_RESERVE))
    torch.cuda.synchronize()
    st, graphs, wss = fresh(), [], [B.workspace(sh, B.CLSA_OP_PAGES_RESERVE) for _ in range(2)]
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(i, st, wss[i])
        graphs.append(g)
    for i in (0, 1, 0, 0, 1):
        graphs[i].replay()
        torch.cuda.synchronize()
        torch.zeros(1000, device="cuda").add_(1)
    assert all(torch.equal(a, b) for a, b in zip((*st[:3], st[4], *st[3]), (*eager[:3], eager[4], *eager[3])))


def test_refusals():
    import torch
    from paper_2606_06467_amd import binding as B
    i = torch.zeros(8, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="one row for each"):
        B.clsa_pages_reserve(_shape(2, 4), [torch.zeros((7, 4), device="cuda")], i, i, i, i, i)
    with pytest.raises(ValueError, match="contiguous"):
        B.clsa_pages_reserve(_shape(2, 4), [torch.zeros((8, 8), device="cuda")[:, ::2]], i, i, i, i, i)
    with pytest.raises(B.ClsaError):
        B.clsa_pages_reserve(_shape(2, 4), [torch.zeros((8, 8), device="cuda")], i, i, i, i, i)  # no workspace
    with pytest.raises(B.ClsaError):
        B.clsa_pages_fork(B.make_shape(2, 1, 64, 1), i, i, i, i)  # not paged
