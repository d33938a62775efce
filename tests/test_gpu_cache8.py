"""GPU parity of the 8-bit cache: appending, and sparse and dense attention from it, against
plain 64-bit references (tests/cache8_util.py)."""
import ctypes

import numpy as np
import pytest

from paper_2606_06467_amd import inputs
from tests import cache8_util as C
from tests import gpu_util as U

pytestmark = pytest.mark.gpu
SCALE = 1 / np.sqrt(128)


def _dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _bf16(bits):
    from paper_2606_06467_amd import binding as B
    return B.bf16_from_bits(bits)


def _shape(batch, n_q, max_len, heads, page=0, top_k=64, group=1, causal=False, **kw):
    from paper_2606_06467_amd import binding as B
    return B.make_shape(batch, n_q, max_len, top_k, q_heads=heads * group, kv_heads=heads,
                        page_size=page, max_pages=max_len // page if page else 0, causal=causal, **kw)


class Pair:
    """K and V caches on both sides."""

    def __init__(self, k, v):
        self.k, self.v = k, v
        self.push()

    def push(self):
        self.k8, self.v8 = _dev(self.k.bytes), _dev(self.v.bytes)
        self.ks, self.vs = _dev(self.k.scale), _dev(self.v.scale)
        self.pt = _dev(self.k.pt)

    def append(self, sh, block, x, start, count):
        """x: (K, V) values [B, n_q, H, D] that bf16 holds; on the GPU and in the references."""
        from paper_2606_06467_amd import binding as B
        bits = [C.bf16(a)[1] for a in x]
        B.clsa_cache_append8(sh, block, _bf16(bits[0]), _bf16(bits[1]), _dev(np.int32(start)),
                             _dev(np.int32(count)), self.pt, self.k8, self.v8, self.ks, self.vs)
        for c, a in ((self.k, x[0]), (self.v, x[1])):
            for b, (s, n) in enumerate(zip(start, count)):
                n = min(max(n, 0), a.shape[1])
                if 0 <= s <= c.max_len and n:
                    n = min(n, c.max_len - s)
                    if n:
                        c.append(b, s, a[b, :n].copy())

    def check(self):
        for c, b8, s in ((self.k, self.k8, self.ks), (self.v, self.v8, self.vs)):
            assert np.array_equal(s.cpu().numpy(), c.scale), "scales"
            assert C.same_bytes(b8.cpu().numpy(), c.bytes), "bytes"


def _random(g, batch, n_q, heads, spread=2.0):
    x = g.standard_normal((2, batch, n_q, heads, 128))
    x *= 2.0 ** (spread * g.standard_normal((2, batch, n_q, heads, 1)))
    return [C.bf16(a)[0] for a in x]


@pytest.mark.parametrize("block,page,heads,n_q", [
    (16, 0, 4, 40), (32, 64, 2, 100), (64, 64, 8, 130), (64, 0, 1, 200), (128, 128, 4, 300),
    (16, 4096, 3, 33), (128, 0, 5, 129), (64, 128, 8, 1)])
def test_append_ragged(block, page, heads, n_q):
    """Several chunks behind one another: starts inside blocks, counts from 0 to n_q."""
    g = np.random.default_rng(block + page + heads + n_q)
    batch, max_len = 5, 1000 if not page else -(-1000 // page) * page
    pt = C.page_table(3, [max_len] * batch, page, max_len) if page else None
    p = Pair(*(C.Cache(batch, max_len, heads, block, page, pt) for _ in "kv"))
    sh = _shape(batch, n_q, max_len, heads, page)
    at = np.array([0, block - 1, 5 * block, 7, max_len - n_q if not page else 2])
    for _ in range(3):
        count = g.integers(0, n_q + 1, size=batch)
        count[0] = n_q
        count = np.minimum(count, max_len - at)
        p.append(sh, block, _random(g, batch, n_q, heads), at, count)
        at = at + count
        p.check()


@pytest.mark.parametrize("block", [16, 64])
def test_append_token_by_token(block):
    """Blocks that grow a token at a time, larger and larger: kept bytes move with the scale."""
    g = np.random.default_rng(block)
    p = Pair(*(C.Cache(2, 150, 2, block) for _ in "kv"))
    sh = _shape(2, 1, 150, 2)
    for j in range(100):
        x = _random(g, 2, 1, 2, 3.0)
        if j % 9 == 8:
            x = [C.bf16(a * 2.0 ** 16)[0] for a in x]  # what was held falls below the least exponent
        p.append(sh, block, x, [j, j + 31], [1, j % 3 > 0])
    p.check()


def test_append_extreme_values():
    """NaN, infinities, zeros, subnormals, the largest values, and a border of the scale."""
    p = Pair(*(C.Cache(1, 256, 2, 64) for _ in "kv"))
    sh = _shape(1, 130, 256, 2)
    x = np.zeros((2, 1, 130, 2, 128))
    x[0, 0, 3, 0, 5], x[0, 0, 4, 0, 6], x[1, 0, 5, 1, 7] = np.nan, np.inf, -np.inf
    x[0, 0, 6] = 448.0                      # exactly held by scale 1
    x[0, 0, 70, 0] = 450.0                  # not by it
    x[1, 0, 7, 0] = 3.38e38
    x[1, 0, 8, 1] = -3.3895313892515355e38  # the largest bf16
    x[1, 0, 75, 0] = 2.0 ** -133            # the least
    x[1, 0, 76, 1] = 3 * 2.0 ** -108
    x = [C.bf16(a)[0] for a in x]
    p.append(sh, 64, x, [10], [130])
    p.check()
    assert p.k.scale[0, 0, 0] == 1.0 and p.k.scale[0, 1, 0] == 2.0 and p.v.scale[0, 1, 0] == 2.0 ** -100
    x = [np.full_like(a, np.nan) for a in x]  # a block of NaN alone keeps its scale
    p.append(sh, 64, x, [140], [20])
    p.check()


def test_append_begins_a_block_afresh():
    """A block that the new tokens begin does not keep the larger scale of what was there."""
    g = np.random.default_rng(1)
    p = Pair(*(C.Cache(1, 128, 2, 32) for _ in "kv"))
    sh = _shape(1, 40, 128, 2)
    p.append(sh, 32, [a * 64 for a in _random(g, 1, 40, 2, 0.5)], [0], [40])
    p.append(sh, 32, _random(g, 1, 40, 2, 0.5), [32], [20])
    p.check()
    assert (p.k.scale[0, 1] < p.k.scale[0, 0]).all()


def test_append_out_of_range():
    from paper_2606_06467_amd import binding as B
    g = np.random.default_rng(2)
    B.clsa_get_device_error()
    for start, count, bits in (([0, 90], [8, 8], 0), ([95, 3], [8, 9], 4), ([-1, 101], [2, 2], 4),
                               ([100, 0], [0, -3], 4), ([100, 5], [0, 0], 0), ([2 ** 31 - 1, 0], [8, 8], 4)):
        p = Pair(*(C.Cache(2, 100, 2, 16) for _ in "kv"))
        p.append(_shape(2, 8, 100, 2), 16, _random(g, 2, 8, 2), start, count)
        p.check()
        assert B.clsa_get_device_error() == bits, (start, count)


def _attend(p, sh, block, q, idx=None, ns=None, lens=None, q_pos=None, with_lse=True):
    import torch
    from paper_2606_06467_amd import binding as B
    qd = _bf16(q)
    out = torch.full(qd.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full(qd.shape[:-1], float("nan"), device="cuda") if with_lse else None
    if idx is not None:
        ws = B.workspace(sh, B.CLSA_OP_ATTN8)
        B.clsa_sparse_attn8(sh, block, qd, p.k8, p.v8, p.ks, p.vs, p.pt, _dev(idx), _dev(ns), out, lse, ws)
    else:
        ws = B.workspace(sh, B.CLSA_OP_DENSE8)
        B.clsa_dense_attn8(sh, block, qd, p.k8, p.v8, p.ks, p.vs, p.pt, _dev(np.int32(lens)), _dev(q_pos),
                           out, lse, ws)
    torch.cuda.synchronize()
    return B.bits_from_bf16(out), lse.cpu().numpy().astype(np.float64) if with_lse else None


def _sets(g, lens, n_q, k, counts=None):
    """Random ascending lists, -1 padded, and as sets."""
    idx = np.full((len(lens), n_q, k), -1, np.int32)
    ns = np.zeros((len(lens), n_q), np.int32)
    sets = []
    for b, n in enumerate(lens):
        sets.append([])
        for t in range(n_q):
            m = min(k, n) if counts is None else min(counts[b][t], n, k)
            s = np.sort(g.choice(n, size=m, replace=False)) if n else np.zeros(0, int)
            idx[b, t, :m] = s
            ns[b, t] = m
            sets[-1].append(s)
    return idx, ns, sets


def _sparse_case(seed, lens, heads, group, k, block, page=0, n_q=1, counts=None, scale=None, with_lse=True):
    g = np.random.default_rng(seed)
    top = max(lens)
    max_len = -(-top // page) * page if page else top
    pt = C.page_table(seed, lens, page, max_len) if page else None
    p = Pair(*(C.filled(seed + i, lens, heads, block, max_len, page, pt) for i in (1, 2)))
    qv, q = C.bf16(g.standard_normal((len(lens), n_q, heads * group, 128)))
    idx, ns, sets = _sets(g, lens, n_q, k, counts)
    kw = {} if scale is None else dict(softmax_scale=scale)
    sh = _shape(len(lens), n_q, max_len, heads, page, k, group, **kw)
    out, lse = _attend(p, sh, block, q, idx, ns, with_lse=with_lse)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, sets, SCALE if scale is None else np.float32(scale)))


@pytest.mark.parametrize("group", [1, 2, 4, 5, 8])
@pytest.mark.parametrize("page", [0, 64])
def test_sparse_groups(group, page):
    _sparse_case(group, (700, 450), 2, group, 300, 32, page)


@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 127, 128, 129, 1000, 8192])
def test_sparse_list_lengths(k):
    _sparse_case(k, (max(40, min(k, 1500)), 40), 2, 4, k, 64)


@pytest.mark.parametrize("block,page", [(16, 16), (16, 0), (32, 128), (128, 0), (128, 128), (64, 4096)])
def test_sparse_blocks(block, page):
    _sparse_case(block + page, (333, 1, 130), 4, 2, 200, block, page)


def test_sparse_empty_and_partial_lists():
    _sparse_case(5, (300, 200, 100), 2, 4, 256, 32, n_q=3,
                 counts=[[0, 1, 256], [33, 0, 31], [64, 65, 0]])


def test_sparse_many_rows():
    """Rows enough that one workgroup takes a row's whole list."""
    g = np.random.default_rng(6)
    counts = [list(g.integers(0, 150, size=300))]
    _sparse_case(6, (400,), 4, 2, 140, 64, n_q=300, counts=counts)


@pytest.mark.parametrize("k,n_q,max_len", [(1030, 1030, 25000), (1500, 1025, 70000), (100, 1040, 25000),
                                           (1100, 1030, 2000)])
def test_sparse_rows_by_stretches(k, n_q, max_len):
    """Over 8192 (row, KV head) pairs: long lists are cut into stretches that all rows take in turn
    (checked on some rows of every kind)."""
    g = np.random.default_rng(k)
    n, heads, block = 2000, 8, 32
    p = Pair(*(C.filled(k + i, (n,), heads, block, max_len) for i in (1, 2)))
    counts = [list(np.where(g.random(n_q) < 0.3, g.integers(0, k + 1, size=n_q), k))]
    counts[0][:5] = [0, 1, k // 8, k // 8 + 1, k - 1]
    qv, q = C.bf16(g.standard_normal((1, n_q, heads, 128)))
    idx, ns, sets = _sets(g, (n,), n_q, k, counts)
    out, lse = _attend(p, _shape(1, n_q, max_len, heads, 0, k), block, q, idx, ns)
    at = [*range(8), *g.integers(0, n_q, size=40), n_q - 1]
    C.check_attention(out[:, at], lse[:, at], C.attention(qv[:, at], p.k, p.v, [[sets[0][t] for t in at]], SCALE))


@pytest.mark.parametrize("scale", [0.0, -0.25, 3.0])
def test_sparse_softmax_scale(scale):
    _sparse_case(7, (300, 200), 2, 4, 128, 64, scale=scale)


def test_sparse_without_lse():
    _sparse_case(8, (300, 200), 2, 4, 200, 64, with_lse=False)


def test_sparse_nan_reaches_the_rows_that_select_it():
    """Token 0 (where padding points) and a neighbour hold NaN: only lists with them see it."""
    g = np.random.default_rng(9)
    p = Pair(*(C.filled(9 + i, (300,), 2, 32, 300) for i in (1, 2)))
    p.k.bytes[0, 0] = 0x7f
    p.v.bytes[0, 0] = 0xff
    p.v.bytes[0, 77, 1, 3] = 0x7f
    p.k.bytes[0, 120, 0, 9] = 0xff
    p.push()
    lists = [[1, 5, 9], [0, 5, 9], [5, 77, 200], [76, 78, 119, 121], list(range(121, 290)), [120], []]
    k = 200
    idx, ns = np.full((1, 7, k), -1, np.int32), np.zeros((1, 7), np.int32)
    for t, s in enumerate(lists):
        idx[0, t, :len(s)], ns[0, t] = s, len(s)
    qv, q = C.bf16(g.standard_normal((1, 7, 8, 128)))
    out, lse = _attend(p, _shape(1, 7, 300, 2, 0, k, 4), 32, q, idx, ns)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, [[np.array(s, int) for s in lists]], SCALE))


def test_sparse_counts_out_of_range_are_clamped():
    from paper_2606_06467_amd import binding as B
    g = np.random.default_rng(10)
    p = Pair(*(C.filled(10 + i, (300, 300), 2, 32, 300) for i in (1, 2)))
    idx, ns, sets = _sets(g, (300, 300), 1, 64)
    ns[0], ns[1] = -5, 70
    B.clsa_get_device_error()
    qv, q = C.bf16(g.standard_normal((2, 1, 2, 128)))
    out, lse = _attend(p, _shape(2, 1, 300, 2, 0, 64), 32, q, idx, ns)
    sets[0][0] = np.zeros(0, int)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, sets, SCALE))
    assert B.clsa_get_device_error() == B.CLSA_DEVERR_N_SEL


@pytest.mark.parametrize("paged", [False, True])
def test_sparse_offsets_past_32_bits(paged):
    """Caches of over 4 GiB whose only numbers are the selected tokens, at the far end."""
    import torch
    from paper_2606_06467_amd import binding as B
    g = np.random.default_rng(11)
    heads, block, k, n = 64, 64, 40, 262080
    batch, page = (3, 0) if not paged else (3, 64)
    k8, v8 = (torch.full((batch * n, heads, 128), 0x7f, dtype=torch.uint8, device="cuda") for _ in "kv")
    ks, vs = (torch.full((batch * n // block, heads), float("nan"), device="cuda") for _ in "kv")
    pt = None
    if paged:  # sequence 0 lies in the last pages
        pt = torch.arange(batch * n // page, dtype=torch.int32).flip(0).view(batch, -1).contiguous()
    idx = np.sort(np.concatenate([[0, n - 1], g.choice(np.arange(1, n - 1), k - 2, replace=False)]))
    kv = np.zeros((2, batch, k, heads, 128))
    row = []
    for b in range(batch):
        at = idx if not paged else (pt[b].numpy()[idx // page].astype(np.int64) * page + idx % page)
        row.append(at if paged else at + b * n)
        byte = np.where((r := g.integers(0, 256, (2, k, heads, 128))) % 128 == 127, r - 1, r).astype(np.uint8)
        k8[torch.from_numpy(row[b]).cuda()] = _dev(byte[0])
        v8[torch.from_numpy(row[b]).cuda()] = _dev(byte[1])
        kv[:, b] = C.VALUES[byte] / 64
        for s in (ks, vs):
            s[torch.from_numpy(row[b] // block).cuda()] = 1 / 64
    qv, q = C.bf16(g.standard_normal((batch, 1, heads, 128)) / 8)
    sh = _shape(batch, 1, n, heads, page, k, softmax_scale=0.05)
    out = torch.zeros((batch, 1, heads, 128), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((batch, 1, heads), device="cuda")
    B.clsa_sparse_attn8(sh, block, _bf16(q), k8, v8, ks, vs, None if pt is None else pt.cuda(),
                        _dev(np.tile(idx.astype(np.int32), (batch, 1, 1))),
                        _dev(np.full((batch, 1), k, np.int32)), out, lse, B.workspace(sh, B.CLSA_OP_ATTN8))
    torch.cuda.synchronize()
    small = [C.Cache(batch, k, heads, 64) for _ in "kv"]
    for c, x in zip(small, kv):
        c.values = lambda x=x: x
    want = C.attention(qv, *small, [[np.arange(k)]] * batch, np.float32(0.05))
    C.check_attention(B.bits_from_bf16(out), lse.cpu().numpy().astype(np.float64), want)


def _dense_case(seed, lens, heads, group, block, page=0, n_q=1, causal=False, tiles=None, max_len=None,
                nan_at=None, of="v"):
    g = np.random.default_rng(seed)
    top = max_len or max(max(lens), 1)
    max_len = -(-top // page) * page if page else top
    pt = C.page_table(seed, lens, page, max_len) if page else None
    p = Pair(*(C.filled(seed + i, lens, heads, block, max_len, page, pt) for i in (1, 2)))
    if nan_at is not None:
        c = getattr(p, of)
        c.bytes[c.at(0, nan_at)][0, 7] = 0x7f
        p.push()
    qv, q = C.bf16(g.standard_normal((len(lens), n_q, heads * group, 128)))
    q_pos = None
    valid = [[n] * n_q for n in lens]
    if causal:
        q_pos = np.array([[n - n_q + t for t in range(n_q)] for n in lens], np.int32)
        valid = [[max(0, n - n_q + t + 1) for t in range(n_q)] for n in lens]
    sh = _shape(len(lens), n_q, max_len, heads, page, 64, group, causal)
    if tiles is not None:
        gm = U._Geometry(len(lens), n_q, len(lens) * n_q, max_len, page.bit_length() - 1,
                         max_len // page if page else 0, 64, int(causal), heads * group, heads, group, SCALE)
        from paper_2606_06467_amd import binding as B
        f = B.lib()._ZN4clsa15dense8_in_tilesERKNS_8GeometryE
        f.restype = ctypes.c_bool
        assert f(ctypes.byref(gm)) == tiles
    out, lse = _attend(p, sh, block, q, lens=lens, q_pos=q_pos)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, [[np.arange(m) for m in v] for v in valid], SCALE))


@pytest.mark.parametrize("page", [0, 64])
def test_dense_lengths(page):
    _dense_case(20 + page, (0, 1, 2, 31, 32, 33, 64, 127, 128, 129, 500), 2, 4, 16, page, max_len=513)


@pytest.mark.parametrize("group,block", [(1, 128), (2, 64), (5, 32), (8, 16)])
def test_dense_groups(group, block):
    _dense_case(30 + group, (900, 333), 2, group, block, 128 if group < 4 else 0)


def test_dense_long_split_over_many_ranges():
    _dense_case(40, (9000,), 1, 4, 64)


@pytest.mark.parametrize("page", [0, 128])
def test_dense_causal_few_rows(page):
    """Some rows before a sequence's first token see nothing."""
    _dense_case(50, (200, 3, 77), 2, 2, 32, page, n_q=9, causal=True, tiles=False)


@pytest.mark.parametrize("lens,heads,group,block,page,n_q,causal", [
    ((700, 520), 4, 2, 64, 64, 300, True), ((600,), 4, 5, 16, 0, 600, True),
    ((4000,), 4, 8, 128, 0, 33, False), ((3000, 1), 2, 4, 32, 64, 100, True)])
def test_dense_tiles(lens, heads, group, block, page, n_q, causal):
    _dense_case(60 + n_q, lens, heads, group, block, page, n_q, causal)


@pytest.mark.parametrize("group,block,page", [(5, 16, 0), (8, 128, 128), (1, 32, 64)])
def test_dense_tiles_of_a_long_context(group, block, page):
    """Few rows over many keys: key ranges joined by the log-sum-exp rule."""
    _dense_case(80 + group, (6000, 3500), 2, group, block, page, 70, True, tiles=True)


@pytest.mark.parametrize("of", ["k", "v"])
def test_dense_tiles_nan_reaches_later_rows_only(of):
    _dense_case(70, (500,), 4, 4, 32, 0, 500, True, nan_at=333, of=of)
    _dense_case(72, (6000,), 2, 4, 32, 0, 70, True, tiles=True, nan_at=5960, of=of)


@pytest.mark.parametrize("of", ["k", "v"])
def test_dense_rows_nan_reaches_later_rows_only(of):
    _dense_case(71, (300,), 2, 4, 32, 0, 6, True, tiles=False, nan_at=297, of=of)


def test_binding_refuses_tensors_that_are_not_contiguous():
    import torch
    from paper_2606_06467_amd import binding as B
    p = Pair(*(C.filled(73 + i, (64,), 2, 32, 64) for i in (1, 2)))
    x = torch.zeros((1, 8, 2, 256), dtype=torch.bfloat16, device="cuda")[..., ::2]
    n = torch.ones(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="v must be contiguous"):
        B.clsa_cache_append8(_shape(1, 8, 64, 2), 32, x.contiguous(), x, n, n, None, p.k8, p.v8, p.ks, p.vs)
    with pytest.raises(ValueError, match="k8 must be a GPU tensor"):
        B.clsa_cache_append8(_shape(1, 8, 64, 2), 32, x.contiguous(), x.contiguous(), n, n, None, p.k8.cpu(),
                             p.v8, p.ks, p.vs)


def test_another_stream():
    """The call's stream: the one given, or the current one."""
    import torch
    from paper_2606_06467_amd import binding as B
    g = np.random.default_rng(74)
    p = Pair(*(C.filled(74 + i, (700,), 2, 32, 700) for i in (1, 2)))
    qv, q = C.bf16(g.standard_normal((1, 1, 8, 128)))
    idx, ns, sets = _sets(g, (700,), 1, 300)
    args = _bf16(q), p.k8, p.v8, p.ks, p.vs, None, _dev(idx), _dev(ns)
    sh = _shape(1, 1, 700, 2, 0, 300, 4)
    want = C.attention(qv, p.k, p.v, sets, SCALE)
    torch.cuda.synchronize()
    for given in (False, True):
        st = torch.cuda.Stream()
        out = torch.zeros((1, 1, 8, 128), dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros((1, 1, 8), device="cuda")
        ws = B.workspace(sh, B.CLSA_OP_ATTN8)
        torch.cuda.synchronize()
        if given:
            B.clsa_sparse_attn8(sh, 32, *args, out, lse, ws, stream=st)
        else:
            with torch.cuda.stream(st):
                B.clsa_sparse_attn8(sh, 32, *args, out, lse, ws)
        st.synchronize()
        C.check_attention(B.bits_from_bf16(out), lse.cpu().numpy().astype(np.float64), want)


@pytest.mark.parametrize("key_exp,query_exp,scale_exp", [(-100, 120, -28), (119, -119, -8)])
@pytest.mark.parametrize("lens,heads,group,n_q,k", [
    ((300, 200), 2, 4, 1, 128), ((400,), 4, 2, 200, 140), ((900, 333), 2, 5, 1, 0), ((200, 77), 2, 2, 9, 0),
    ((3500,), 2, 5, 70, 0)])
def test_logits_of_large_and_small_factors(lens, heads, group, n_q, k, key_exp, query_exp, scale_exp):
    """Logits are finite where the products of the queries with the bytes alone are not (lists of k
    tokens; k = 0: dense, the last case in key tiles)."""
    g = np.random.default_rng(n_q + k)
    p = Pair(*(C.filled(90 + i, lens, heads, 32, max(lens)) for i in (1, 2)))
    p.k.scale[:] = 2.0 ** key_exp
    p.push()
    qv, q = C.bf16(g.standard_normal((len(lens), n_q, heads * group, 128)) * 2.0 ** query_exp)
    scale = 2.0 ** scale_exp
    sh = _shape(len(lens), n_q, max(lens), heads, 0, k or 64, group, softmax_scale=scale)
    if k:
        idx, ns, sets = _sets(g, lens, n_q, k)
        out, lse = _attend(p, sh, 32, q, idx, ns)
    else:
        sets = [[np.arange(n)] * n_q for n in lens]
        out, lse = _attend(p, sh, 32, q, lens=lens)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, sets, scale))


class _Plan8(ctypes.Structure):
    """The library's cut of attention by rows (csrc/clsa_internal.h)."""
    _fields_ = [(n, ctypes.c_int) for n in ("heads", "waves", "splits", "span")]


def _geometry(batch, n_q, max_len, heads, group, page=0, top_k=64, causal=False):
    return U._Geometry(batch, n_q, batch * n_q, max_len, page.bit_length() - 1, max_len // page if page else 0,
                       top_k, int(causal), heads * group, heads, group, SCALE)


def _plan(keys, dense, *a, **kw):
    from paper_2606_06467_amd import binding as B
    f = B.lib()._ZN4clsa12plan_splits8ERKNS_8GeometryEib
    f.restype = _Plan8
    p = f(ctypes.byref(_geometry(*a, **kw)), ctypes.c_int(keys), ctypes.c_bool(dense))
    return p.heads, p.waves, p.splits


def _tile_plan(*a, **kw):
    """Whether dense attention runs over key tiles, and in how many key ranges it would."""
    from paper_2606_06467_amd import binding as B
    gm, n, span = _geometry(*a, **kw), ctypes.c_int(), ctypes.c_int()
    f = B.lib()._ZN4clsa15dense8_in_tilesERKNS_8GeometryE
    f.restype = ctypes.c_bool
    B.lib()._ZN4clsa14tile_attn_planERKNS_8GeometryEiRiS3_(ctypes.byref(gm), ctypes.c_int(128), ctypes.byref(n),
                                                         ctypes.byref(span))
    return f(ctypes.byref(gm)), n.value


def _widen_capacity(p, max_len):
    """The caches in a larger capacity, what is new in it NaN; the references keep the small one."""
    import torch
    if p.k.page:
        pt = torch.full((len(p.k.pt), max_len // p.k.page), -1, dtype=torch.int32, device="cuda")
        pt[:, :p.pt.shape[1]] = p.pt
        p.pt = pt
        return
    for name, n, fill in (("k8", max_len, 0x7f), ("v8", max_len, 0x7f), ("ks", -(-max_len // p.k.block), float("nan")),
                          ("vs", -(-max_len // p.k.block), float("nan"))):
        x = getattr(p, name)
        y = torch.full((x.shape[0], n, *x.shape[2:]), fill, dtype=x.dtype, device="cuda")
        y[:, :x.shape[1]] = x
        setattr(p, name, y)


@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("group,heads", [(1, 4), (2, 4), (4, 8), (5, 4), (8, 4)])
def test_dense_four_heads_a_workgroup(group, heads, page):
    """Single tokens over capacities large enough that a workgroup takes four KV heads: key ranges of
    one to several steps, ragged lengths, rows without keys, and NaN in one head of one sequence."""
    g = np.random.default_rng(100 + group)
    lens, block, capacity = (0, 1, 333, 2100, 640, 3001, 1280, 641, 0), 32, 131072 // heads
    batch, small = len(lens), 3008
    heads_, waves, splits = _plan(capacity, True, batch, 1, capacity, heads, group, page)
    assert (heads_, waves) == (4, 1) and splits > 8
    pt = C.page_table(group, lens, page, small) if page else None
    p = Pair(*(C.filled(100 + group + i, lens, heads, block, small, page, pt) for i in (1, 2)))
    p.k.bytes[p.k.at(3, 2040)][1, 7] = 0xff
    p.v.bytes[p.v.at(5, 70)][3, 9] = 0x7f
    p.push()
    _widen_capacity(p, capacity)
    qv, q = C.bf16(g.standard_normal((batch, 1, heads * group, 128)))
    out, lse = _attend(p, _shape(batch, 1, capacity, heads, page, 64, group), block, q, lens=lens)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, [[np.arange(n)] for n in lens], SCALE))


def _sampled(p, sh, block, qv, q, lens, q_pos, valid, at):
    out, lse = _attend(p, sh, block, q, lens=lens, q_pos=q_pos)
    want = C.attention(qv[:, at], p.k, p.v, [[np.arange(v[t]) for t in at] for v in valid], SCALE)
    C.check_attention(out[:, at], lse[:, at], want)


@pytest.mark.parametrize("group,heads,n_q,lens,page,block,causal", [
    (8, 4, 701, (701, 0, 433), 0, 16, True), (8, 4, 701, (701, 0, 433), 64, 64, True),
    (5, 4, 1303, (1303, 700, 0), 128, 32, True), (5, 4, 1303, (1303, 700, 0), 0, 128, True),
    (4, 8, 1025, (1100, 1), 0, 64, False), (2, 8, 1040, (1111, 64, 1000, 65), 16, 16, True),
    (1, 8, 2100, (2100, 1500, 700, 2000), 0, 32, True)])
@pytest.mark.parametrize("of", [None, "k", "v"])
def test_dense_tiles_in_one_range(group, heads, n_q, lens, page, block, causal, of):
    """Whole prompts: tiles whose workgroups write their rows' results themselves (checked on some rows
    of every kind); with a NaN token in the first sequence."""
    g = np.random.default_rng(n_q + page)
    batch, max_len = len(lens), -(-max(lens) // (page or 1)) * (page or 1)
    assert _tile_plan(batch, n_q, max_len, heads, group, page, 64, causal) == (True, 1)
    pt = C.page_table(n_q, lens, page, max_len) if page else None
    p = Pair(*(C.filled(n_q + i, lens, heads, block, max_len, page, pt) for i in (1, 2)))
    if of:
        c = getattr(p, of)
        c.bytes[c.at(0, 333)][heads - 1, 7] = 0x7f
        p.push()
    qv, q = C.bf16(g.standard_normal((batch, n_q, heads * group, 128)))
    q_pos, valid = None, [[n] * n_q for n in lens]
    if causal:
        q_pos = np.array([[n - n_q + t for t in range(n_q)] for n in lens], np.int32)
        valid = [[max(0, n - n_q + t + 1) for t in range(n_q)] for n in lens]
    # the first sequence's rows on both sides of the NaN token, the first and last ones, some more
    nan_row = 333 - (lens[0] - n_q)
    at = sorted({0, 1, 31, 32, 63, 64, nan_row - 1, nan_row, n_q - 2, n_q - 1, *g.integers(0, n_q, size=8).tolist()})
    _sampled(p, _shape(batch, n_q, max_len, heads, page, 64, group, causal), block, qv, q, lens, q_pos, valid, at)


@pytest.mark.parametrize("group,heads,n_q,lens,page,causal", [
    (2, 4, 300, (700, 520), 64, True), (5, 4, 600, (600,), 0, True), (8, 4, 33, (4000,), 0, False),
    (4, 2, 100, (3000, 1), 64, True), (4, 4, 500, (500,), 0, True)])
@pytest.mark.parametrize("of", [None, "k", "v"])
def test_dense_near_the_border_of_both_forms(group, heads, n_q, lens, page, causal, of):
    """Shapes whose two prices lie near each other, in the form that the library takes for them."""
    g = np.random.default_rng(n_q)
    batch, max_len = len(lens), -(-max(lens) // (page or 1)) * (page or 1)
    pt = C.page_table(n_q, lens, page, max_len) if page else None
    p = Pair(*(C.filled(n_q + i, lens, heads, 32, max_len, page, pt) for i in (1, 2)))
    nan_at = lens[0] - n_q // 2
    if of:
        c = getattr(p, of)
        c.bytes[c.at(0, nan_at)][0, 100] = 0xff
        p.push()
    qv, q = C.bf16(g.standard_normal((batch, n_q, heads * group, 128)))
    q_pos, valid = None, [[n] * n_q for n in lens]
    if causal:
        q_pos = np.array([[n - n_q + t for t in range(n_q)] for n in lens], np.int32)
        valid = [[max(0, n - n_q + t + 1) for t in range(n_q)] for n in lens]
    nan_row = n_q - n_q // 2
    at = sorted({0, 1, 31, 32, nan_row - 1, nan_row, n_q - 1, *g.integers(0, n_q, size=8).tolist()})
    _sampled(p, _shape(batch, n_q, max_len, heads, page, 64, group, causal), 32, qv, q, lens, q_pos, valid, at)


@pytest.mark.parametrize("page,block", [(16, 16), (64, 32), (256, 128)])
def test_sparse_paged_many_rows(page, block):
    """One wave a workgroup over pages in any order: lists of many steps that end anywhere in one."""
    g = np.random.default_rng(page)
    n_q, heads, group, k, lens = 200, 4, 2, 900, (1500,)
    max_len = -(-1500 // page) * page
    assert _plan(k, False, 1, n_q, max_len, heads, group, page, k) == (1, 1, 1)
    counts = [list(g.integers(0, k + 1, size=n_q))]
    counts[0][:12] = [0, 1, 31, 32, 33, 63, 64, 65, 95, 96, 97, k]
    _sparse_case(page, lens, heads, group, k, block, page, n_q, counts)


@pytest.mark.parametrize("k,n_q,capacity", [(1030, 1030, 25088), (1500, 1025, 70016)])
@pytest.mark.parametrize("page", [64, 4096])
def test_sparse_paged_rows_by_stretches(page, k, n_q, capacity):
    """Lists cut into stretches, over pages (checked on some rows of every kind)."""
    g = np.random.default_rng(k + page)
    n, heads, block = 2000, 8, 32
    capacity = -(-capacity // page) * page
    assert _plan(k, False, 1, n_q, capacity, heads, 1, page, k)[2] > 1
    pt = C.page_table(k, (n,), page, capacity)
    p = Pair(*(C.filled(k + i, (n,), heads, block, capacity, page, pt) for i in (1, 2)))
    counts = [list(np.where(g.random(n_q) < 0.3, g.integers(0, k + 1, size=n_q), k))]
    counts[0][:5] = [0, 1, k // 8, k // 8 + 1, k - 1]
    qv, q = C.bf16(g.standard_normal((1, n_q, heads, 128)))
    idx, ns, sets = _sets(g, (n,), n_q, k, counts)
    out, lse = _attend(p, _shape(1, n_q, capacity, heads, page, k), block, q, idx, ns)
    at = [*range(8), *g.integers(0, n_q, size=40), n_q - 1]
    C.check_attention(out[:, at], lse[:, at], C.attention(qv[:, at], p.k, p.v, [[sets[0][t] for t in at]], SCALE))


@pytest.mark.parametrize("page,block,k", [(16, 16, 1000), (64, 32, 2048), (128, 128, 1777), (64, 64, 8192)])
@pytest.mark.parametrize("heads", [1, 8])
def test_sparse_paged_long_lists(page, block, k, heads):
    """Few rows over pages in any order: several steps a wave, or several ranges, ending anywhere."""
    n = 3000 if k < 8192 else 8500
    counts = [[m] for m in (k, k - 1, 0, 1, 255, 256, 257, 511, 513, k // 2 + 3, 97)]
    _sparse_case(k + heads, [n] * len(counts), heads, 2, k, block, page, 1, counts)


def test_sparse_paged_long_lists_of_several_rows():
    """2 to 31 rows a sequence, as in checking several proposed tokens at once."""
    g = np.random.default_rng(7)
    _sparse_case(77, (2500, 2200, 1999), 2, 4, 1200, 64, 64, 5, [list(g.integers(0, 1201, size=5)) for _ in range(3)])
    _sparse_case(78, (2500, 2200), 2, 5, 700, 32, 0, 31, [list(g.integers(0, 701, size=31)) for _ in range(2)])


@pytest.mark.parametrize("lens,heads,group,n_q,k,page", [
    ((300, 260), 2, 4, 1, 256, 0), ((700, 600), 1, 1, 1, 600, 64), ((500,), 2, 2, 400, 450, 0),
    ((500, 400), 4, 5, 100, 400, 64), ((400, 300), 2, 8, 1, 0, 0), ((900, 800), 2, 5, 1, 0, 64),
    ((600, 200), 2, 8, 7, 0, 0)])
def test_weights_keep_16_bits(lens, heads, group, n_q, k, page):
    """Logits that fp32 holds exactly, so that the weights' rounding is what the outputs show beside their own.

    A weight is off by 2^-8 of what its first piece left, 2^-16 of it; the exponent's product with the scale
    by 2^-24 of up to 40, twice with the maximum's, and the exponential by a few 2^-24 (2^-17 in all), of
    which the sum of weights carries as much; both sums over n keys by n 2^-24, the merging by 2^-20."""
    g = np.random.default_rng(heads + n_q + k)
    max_len = -(-max(lens) // page) * page if page else max(lens)
    pt = C.page_table(n_q, lens, page, max_len) if page else None
    p = Pair(*(C.filled(95 + i, lens, heads, 32, max_len, page, pt) for i in (1, 2)))
    held = (p.k.bytes & 0x7f) != 0x7f
    p.k.bytes[held] = C.encode(g.integers(-4, 5, size=p.k.bytes.shape).astype(np.float64))[held]
    p.k.scale[:] = 1.0
    p.push()
    qv = g.integers(-4, 5, size=(len(lens), n_q, heads * group, 128)).astype(np.float64)
    q, scale = C.bf16(qv)[1], 2.0 ** -5
    sh = _shape(len(lens), n_q, max_len, heads, page, k or 64, group, softmax_scale=scale)
    if k:
        idx, ns, sets = _sets(g, lens, n_q, k)
        out = _attend(p, sh, 32, q, idx, ns, with_lse=False)[0]
    else:
        assert not _tile_plan(len(lens), n_q, max_len, heads, group, page)[0]
        sets = [[np.arange(n)] * n_q for n in lens]
        out = _attend(p, sh, 32, q, lens=lens, with_lse=False)[0]
    out = inputs.f32_from_bf16_bits(out).astype(np.float64)
    for b, n in enumerate(lens):
        kb, vb = p.k.rows(b, n), p.v.rows(b, n)
        for t in range(0, n_q, 1 if n_q < 50 else 17):
            for h in range(heads * group):
                z = kb[sets[b][t], h // group] @ qv[b, t, h] * scale
                w = np.exp(z - z.max())
                w /= w.sum()
                v = vb[sets[b][t], h // group]
                o = w @ v
                tol = w @ np.abs(v) * (2.0 ** -16 + 2 * 2.0 ** -17 + 2 * len(z) * 2.0 ** -24 + 2.0 ** -20) + \
                    2.0 ** -8 * np.abs(o) * 1.001
                off = np.abs(out[b, t, h] - o) / tol
                assert off.max() <= 1.0, (b, t, h, off.max())


@pytest.mark.parametrize("value_exp", [-100, 96])
@pytest.mark.parametrize("lens,heads,group,n_q,k", [
    ((300, 200), 2, 4, 1, 128), ((400,), 4, 5, 200, 140), ((900, 333), 2, 8, 1, 0), ((3500,), 2, 5, 70, 0)])
def test_smallest_and_large_values(lens, heads, group, n_q, k, value_exp):
    """Value scales at their least, and as large as sums of values may be (k = 0: dense, the last in tiles)."""
    g = np.random.default_rng(n_q + k)
    p = Pair(*(C.filled(97 + i, lens, heads, 32, max(lens)) for i in (1, 2)))
    p.v.scale[:] = 2.0 ** value_exp
    p.push()
    qv, q = C.bf16(g.standard_normal((len(lens), n_q, heads * group, 128)))
    sh = _shape(len(lens), n_q, max(lens), heads, 0, k or 64, group)
    if k:
        idx, ns, sets = _sets(g, lens, n_q, k)
        out, lse = _attend(p, sh, 32, q, idx, ns)
    else:
        sets = [[np.arange(n)] * n_q for n in lens]
        out, lse = _attend(p, sh, 32, q, lens=lens)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, sets, SCALE))


@pytest.mark.parametrize("scale", [0.0, -0.25, 3.0])
@pytest.mark.parametrize("lens,heads,group,n_q,page,tiles", [
    ((300, 0, 201), 3, 4, 1, 0, False), ((2100, 1999), 3, 5, 4, 64, False), ((3500, 2900), 3, 2, 70, 64, True)])
def test_dense_softmax_scale(lens, heads, group, n_q, page, tiles, scale):
    g = np.random.default_rng(n_q)
    max_len = -(-max(lens) // page) * page if page else max(lens)
    assert _tile_plan(len(lens), n_q, max_len, heads, group, page, 64, True)[0] == tiles
    pt = C.page_table(n_q, lens, page, max_len) if page else None
    p = Pair(*(C.filled(98 + i, lens, heads, 32, max_len, page, pt) for i in (1, 2)))
    qv, q = C.bf16(g.standard_normal((len(lens), n_q, heads * group, 128)))
    q_pos = np.array([[n - n_q + t for t in range(n_q)] for n in lens], np.int32)
    sets = [[np.arange(max(0, n - n_q + t + 1)) for t in range(n_q)] for n in lens]
    sh = _shape(len(lens), n_q, max_len, heads, page, 64, group, True, softmax_scale=scale)
    out, lse = _attend(p, sh, 32, q, lens=lens, q_pos=q_pos)
    C.check_attention(out, lse, C.attention(qv, p.k, p.v, sets, np.float32(scale)))


@pytest.mark.parametrize("n_q,k,capacity", [(1030, 1500, 70016), (1, 2048, 4096), (40, 300, 4096)])
def test_captured_lists(n_q, k, capacity):
    """Lists in stretches, in ranges and whole, replayed between eager calls with other queries and lists."""
    import torch
    from paper_2606_06467_amd import binding as B
    g = np.random.default_rng(k)
    n, heads = 3000, 8
    p = Pair(*(C.filled(k + i, (n,), heads, 64, n) for i in (1, 2)))
    _widen_capacity(p, capacity)
    sh = _shape(1, n_q, capacity, heads, 0, k)
    bufs = []
    for _ in "ge":
        q = torch.zeros((1, n_q, heads, 128), dtype=torch.bfloat16, device="cuda")
        bufs.append((q, torch.full((1, n_q, k), -1, dtype=torch.int32, device="cuda"),
                     torch.zeros((1, n_q), dtype=torch.int32, device="cuda"), torch.zeros_like(q),
                     torch.zeros((1, n_q, heads), device="cuda"), B.workspace(sh, B.CLSA_OP_ATTN8)))

    def call(q, idx, ns, out, lse, ws):
        B.clsa_sparse_attn8(sh, 64, q, p.k8, p.v8, p.ks, p.vs, None, idx, ns, out, lse, ws)

    call(*bufs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*bufs[0])
    for _ in range(3):
        idx, ns, _ = _sets(g, (n,), n_q, k, [list(g.integers(0, k + 1, size=n_q))])
        q = _bf16(C.bf16(g.standard_normal((1, n_q, heads, 128)))[1])
        for b in bufs:
            b[0].copy_(q)
            b[1].copy_(torch.from_numpy(idx))
            b[2].copy_(torch.from_numpy(ns))
        graph.replay()
        call(*bufs[1])
        torch.cuda.synchronize()
        for a, b in zip(bufs[0][3:5], bufs[1][3:5]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
