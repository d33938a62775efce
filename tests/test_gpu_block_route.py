"""GPU parity of block routing (means of index keys, choice of blocks) against plain 64-bit
references, and of the whole path: projection, 8-bit cache, block routing, attention."""
import numpy as np
import pytest

from paper_2606_06467_amd import inputs
from tests import cache8_util as C

pytestmark = pytest.mark.gpu


def _dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _bf16(bits):
    from paper_2606_06467_amd import binding as B
    return B.bf16_from_bits(bits)


def _shape(batch, n_q, max_len, top_k, page=0, causal=False, **kw):
    from paper_2606_06467_amd import binding as B
    return B.make_shape(batch, n_q, max_len, top_k, page_size=page,
                        max_pages=max_len // page if page else 0, causal=causal, **kw)


def _rows(batch, max_len, page, pt, per):
    """Row of each (sequence, unit) in a cache of units of `per` tokens, -1 where it has none."""
    units = -(-max_len // per)
    if not page:
        return np.arange(batch * units).reshape(batch, units)
    c = np.arange(units) * per
    r = pt[:, c // page].astype(np.int64) * (page // per) + c % page // per
    return np.where(pt[:, c // page] < 0, -1, r)


@pytest.mark.parametrize("block,page,n_q", [(16, 0, 40), (32, 64, 100), (64, 64, 1), (64, 0, 200), (128, 128, 257)])
def test_means(block, page, n_q):
    """Only blocks whose last token is new are written."""
    import torch
    from paper_2606_06467_amd import binding as B
    g = np.random.default_rng(block + n_q)
    batch, max_len = 6, 1024 if page else 1000
    pt = C.page_table(1, [max_len] * batch, page, max_len) if page else None
    tok = _rows(batch, max_len, page, pt, 1)
    x, bits = C.bf16(g.standard_normal((tok.size, 256)) * 2.0 ** g.integers(-6, 7, size=(tok.size, 1)))
    blk = _rows(batch, max_len, page, pt, block)
    start = np.array([0, block - 1, 3 * block, 5, max_len - min(n_q, 7), max_len], np.int32)
    count = np.minimum(np.array([n_q, 1, n_q, n_q // 2, n_q, 0]), max_len - start).astype(np.int32)
    means = np.full((blk.size, 256), 0x1234, np.uint16)
    md = _bf16(means)
    B.clsa_block_means(_shape(batch, n_q, max_len, 64, page), block, _bf16(bits), _dev(start), _dev(count),
                       _dev(pt), md)
    torch.cuda.synchronize()
    for b in range(batch):
        for c in range(max_len // block):
            if start[b] < (c + 1) * block <= start[b] + count[b]:
                m = x[tok[b, c * block:(c + 1) * block]].sum(0) / block
                means[blk[b, c]] = C.bf16(m)[1]
    assert np.array_equal(B.bits_from_bf16(md), means)


def _topk(sh, block, q, means, lens, q_pos=None, pt=None, fill=-7, shift=0):
    """shift: elements by which the lists miss their 16 bytes."""
    import torch
    from paper_2606_06467_amd import binding as B
    rows = sh.batch * sh.n_q
    buf = torch.full(((rows + 2) * sh.top_k + shift,), fill, dtype=torch.int32, device="cuda")
    buf = buf[shift:].view(rows + 2, sh.top_k)
    nb = torch.full((rows + 2,), fill, dtype=torch.int32, device="cuda")
    ws = B.workspace(sh, B.CLSA_OP_BLOCK_TOPK, block)
    ws.fill_(0xff)
    B.clsa_block_topk(sh, block, _bf16(q), _bf16(means), _dev(pt), _dev(np.int32(lens)), _dev(q_pos),
                      buf[1:rows + 1], nb[1:rows + 1], ws)
    torch.cuda.synchronize()
    assert (buf[[0, -1]] == fill).all() and (nb[[0, -1]] == fill).all()
    return (buf[1:-1].cpu().numpy().reshape(sh.batch, sh.n_q, -1),
            nb[1:-1].cpu().numpy().reshape(sh.batch, sh.n_q))


def _check(sh, block, qv, mv, valid, got):
    """mv[b]: the means of sequence b's blocks."""
    idx, ns = got
    for b in range(sh.batch):
        for t in range(sh.n_q):
            want, n = C.route(qv[b, t], mv[b], valid[b][t], block, sh.top_k)
            assert ns[b, t] == n, (b, t, ns[b, t], n)
            assert np.array_equal(idx[b, t], want), (b, t)


def _case(seed, lens, block, top_k, page=0, n_q=1, causal=False, tweak=None, max_len=None, shift=0):
    g = np.random.default_rng(seed)
    batch, top = len(lens), max_len or max(max(lens), 1)
    max_len = -(-top // page) * page if page else top
    pt = C.page_table(seed, lens, page, max_len) if page else None
    blk = _rows(batch, max_len, page, pt, block)
    # what is not complete holds NaN
    mv = np.full((max(blk.size, blk.max() + 1), 256), np.nan)
    for b, n in enumerate(lens):
        mv[blk[b, :n // block]] = g.standard_normal((n // block, 256)) / 64
    qv = g.standard_normal((batch, n_q, 256)) / 8
    if tweak:
        tweak(g, qv, mv, blk)
    (qv, q), (mv, m) = C.bf16(qv), C.bf16(mv)
    q_pos, valid = None, [[n] * n_q for n in lens]
    if causal:
        q_pos = np.array([[n - n_q + t for t in range(n_q)] for n in lens], np.int32)
        valid = [[max(0, n - n_q + t + 1) for t in range(n_q)] for n in lens]
    sh = _shape(batch, n_q, max_len, top_k, page, causal)
    got = _topk(sh, block, q, m, lens, q_pos, pt, shift=shift)
    _check(sh, block, qv, [mv[np.maximum(blk[b], 0)] for b in range(batch)], valid, got)


@pytest.mark.parametrize("block,page,top_k", [(16, 0, 64), (16, 16, 16), (32, 64, 512), (64, 64, 128),
                                              (64, 0, 2048), (128, 128, 1024), (128, 0, 8192)])
def test_single_tokens(block, page, top_k):
    """From no key to more blocks than are chosen, ends inside a block and on its border."""
    _case(block + top_k, (0, 1, block - 1, block, block + 1, 5 * block, top_k, top_k + 1, top_k + block,
                          7 * top_k + 3, 40 * block + 5), block, top_k, page)


@pytest.mark.parametrize("block,page,top_k,n_q,lens", [
    (16, 0, 64, 100, (700, 90)), (64, 64, 256, 33, (3000, 10)), (32, 128, 512, 200, (2000,)),
    (128, 0, 128, 17, (1500, 1400)), (64, 0, 2048, 64, (9000,))])
def test_causal_rows(block, page, top_k, n_q, lens):
    """Rows of a chunk: each its own block, none of the later ones; some rows see nothing."""
    _case(block + n_q, lens, block, top_k, page, n_q, True)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_lists_off_16_bytes(shift):
    _case(shift, (0, 7, 64, 65, 300, 2000), 16, 48, shift=shift)


def _same(g, qv, mv, blk):
    mv[:] = mv[blk[0, 0]]


@pytest.mark.parametrize("lens,page", [((262144, 200000), 0), ((100000, 131072), 64), ((65536, 33000), 0)])
def test_many_blocks(lens, page):
    """Up to the largest capacity: 4096, 8192 and 16384 blocks of a sequence."""
    _case(3, lens, 16, 512, page)


@pytest.mark.parametrize("lens,n_q", [((262144,), 3), ((120000,), 20), ((65536,), 20)])
def test_many_blocks_alike(lens, n_q):
    """Thousands of equal scores: the lowest blocks."""
    _case(5, lens, 16, 8192, 0, n_q, True, _same)


def _zero_query(g, qv, mv, blk):
    qv[:] = 0


def _few_levels(g, qv, mv, blk):
    mv[:] = g.integers(-1, 2, size=mv.shape)
    qv[:] = g.integers(-1, 2, size=qv.shape) * (g.random(qv.shape) < 0.05)


def _near(g, qv, mv, blk):
    """Scores whose differences fp32 cannot hold: large parts that cancel, small ones that decide."""
    qv[..., 0], qv[..., 1] = 256.0, 256.0
    mv[:, 0], mv[:, 1] = 128.0, -128.0
    mv[:, 2:] = g.integers(-2, 3, size=(len(mv), 254)) * 2.0 ** -14
    qv[..., 2:] = 2.0 ** -10


def _infinite(g, qv, mv, blk):
    qv[..., 5] = 1.0
    mv[blk[0, 3], 5], mv[blk[0, 11], 5], mv[blk[0, 6], 5] = np.inf, -np.inf, np.inf


@pytest.mark.parametrize("tweak", [_same, _zero_query, _few_levels, _near, _infinite])
@pytest.mark.parametrize("n_q", [1, 40])
def test_scores_next_to_one_another(tweak, n_q):
    """Exact ties go to the lowest block, near ones to the larger exact score."""
    with np.errstate(invalid="ignore"):
        _case(n_q, (6400, 3000), 32, 640, 0, n_q, n_q > 1, tweak)


def test_lengths_out_of_range_are_clamped():
    from paper_2606_06467_amd import binding as B
    g = np.random.default_rng(4)
    B.clsa_get_device_error()
    (qv, q), (mv, m) = C.bf16(g.standard_normal((3, 1, 256))), C.bf16(g.standard_normal((3, 16, 256)))
    sh = _shape(3, 1, 256, 64)
    got = _topk(sh, 16, q, m, [-4, 257, 100])
    _check(sh, 16, qv, mv, [[0], [256], [100]], got)
    assert B.clsa_get_device_error() == B.CLSA_DEVERR_SEQ_LEN


class Serving:
    """Buffers of a serving program: projection, caches, block routing and attention."""

    def __init__(self, seed, batch, n_q, max_len, block, top_k, page, layers=2, heads=4, group=4):
        import torch
        from paper_2606_06467_amd import binding as B
        self.B, self.g = B, np.random.default_rng(seed)
        self.batch, self.n_q, self.block, self.layers, self.heads = batch, n_q, block, layers, heads
        self.kw = dict(q_heads=heads * group, kv_heads=heads)
        self.sh = _shape(batch, n_q, max_len, top_k, page, True, **self.kw)
        self.pt = C.page_table(seed, [max_len] * batch, page, max_len) if page else None
        rows = (batch, max_len) if not page else (batch * max_len // page, page)
        blocks = (rows[0], -(-rows[1] // block))
        z = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
        self.d_pt = _dev(self.pt)
        self.k8, self.v8 = (z(*rows, heads, 128, dtype=torch.uint8) for _ in "kv")
        self.ks, self.vs = (z(*blocks, heads) for _ in "kv")
        self.k_idx = z(*rows, 256, dtype=torch.bfloat16)
        self.means = z(*blocks, 256, dtype=torch.bfloat16)
        self.d_model = 512
        self.w = _bf16(C.bf16(self.g.standard_normal((512 + 2 * heads * 128, self.d_model)) / 16)[1])
        self.h = z(batch, n_q, self.d_model, dtype=torch.bfloat16)
        self.q_idx = z(batch, n_q, 256, dtype=torch.bfloat16)
        self.q = z(layers, batch, n_q, heads * group, 128, dtype=torch.bfloat16)
        self.out = z(layers, batch, n_q, heads * group, 128, dtype=torch.bfloat16)
        self.lse = z(layers, batch, n_q, heads * group)
        self.dense, self.dense_lse = torch.zeros_like(self.out[0]), torch.zeros_like(self.lse[0])
        self.idx = z(batch, n_q, top_k, dtype=torch.int32)
        self.n_sel = z(batch, n_q, dtype=torch.int32)
        self.start, self.count, self.lens = (z(batch, dtype=torch.int32) for _ in range(3))
        self.pos = z(batch, n_q, dtype=torch.int32)
        self.ws = [B.workspace(self.sh, B.CLSA_OP_BLOCK_TOPK, block), B.workspace(self.sh, B.CLSA_OP_ATTN8),
                   B.workspace(self.sh, B.CLSA_OP_DENSE8), B.workspace(self.sh, B.CLSA_OP_PROJECT8)]
        self.at = np.zeros(batch, np.int64)

    def feed(self, count):
        """New tokens of every sequence: hidden states, queries and positions."""
        import torch
        g = self.g
        self.h.copy_(_bf16(C.bf16(g.standard_normal(tuple(self.h.shape)))[1]))
        self.q.copy_(_bf16(C.bf16(g.standard_normal(tuple(self.q.shape)))[1]))
        count = np.asarray(count)
        self.start.copy_(torch.from_numpy(self.at.astype(np.int32)))
        self.count.copy_(torch.from_numpy(count.astype(np.int32)))
        self.lens.copy_(torch.from_numpy((self.at + count).astype(np.int32)))
        pos = self.at[:, None] + np.arange(self.n_q)
        pos = np.where(np.arange(self.n_q) < count[:, None], pos, -1)  # rows behind the last one
        self.pos.copy_(torch.from_numpy(pos.astype(np.int32)))
        self.at = self.at + count
        return pos

    def step(self):
        B, sh, n = self.B, self.sh, self.block
        B.clsa_project_append8(sh, n, self.d_model, self.h, self.w, self.start, self.count, self.d_pt,
                               self.q_idx, self.k_idx, self.k8, self.v8, self.ks, self.vs, self.ws[3])
        B.clsa_block_means(sh, n, self.k_idx, self.start, self.count, self.d_pt, self.means)
        B.clsa_block_topk(sh, n, self.q_idx, self.means, self.d_pt, self.lens, self.pos, self.idx, self.n_sel,
                          self.ws[0])
        for l in range(self.layers):
            B.clsa_sparse_attn8(sh, n, self.q[l], self.k8, self.v8, self.ks, self.vs, self.d_pt, self.idx,
                                self.n_sel, self.out[l], self.lse[l], self.ws[1])
        B.clsa_dense_attn8(sh, n, self.q[0], self.k8, self.v8, self.ks, self.vs, self.d_pt, self.lens, self.pos,
                           self.dense, self.dense_lse, self.ws[2])

    def new_rows(self):
        """K and V rows of the step's tokens, by the bf16 projection: [batch, n_q, heads, 128]."""
        import torch
        B = self.B
        order = torch.arange(self.n_q, dtype=torch.int32, device="cuda").repeat(self.batch, 1)
        rows = [torch.zeros(self.batch, self.n_q, *s, dtype=torch.bfloat16, device="cuda")
                for s in ((256,), (256,), (self.heads, 128), (self.heads, 128))]
        B.clsa_project_append(_shape(self.batch, self.n_q, self.n_q, self.sh.top_k, 0, True, **self.kw),
                              self.d_model, self.h, self.w, order, None, *rows)
        return rows

    def results(self):
        return [self.k8, self.v8, self.ks, self.vs, self.means, self.idx, self.n_sel, self.out, self.lse,
                self.dense, self.dense_lse]


@pytest.mark.parametrize("page,block", [(0, 32), (64, 16)])
def test_serving_steps(page, block):
    """A prompt and single tokens through the whole path, each step against the references fed with
    the projection's rows."""
    import torch
    from paper_2606_06467_amd import binding as B
    s = {n: Serving(7, 3, n, 256, block, 4 * block, page) for n in (70, 1)}
    one, many = s[1], s[70]
    for name in ("k8", "v8", "ks", "vs", "k_idx", "means", "w", "d_pt", "pt"):
        setattr(one, name, getattr(many, name))
    ref = [C.Cache(3, 256, 4, block, page, many.pt, fill=0) for _ in "kv"]
    for c in ref:
        c.scale[:] = 0
    for step, (prog, count) in enumerate([(many, [70, 33, 0]), (many, [64, 1, 70]), (one, [1, 1, 1]),
                                          (one, [1, 0, 1]), (one, [1, 1, 1])]):
        if step:
            prog.at = last.at
        last = prog
        first = prog.at.copy()
        pos = prog.feed(count)
        prog.step()
        torch.cuda.synchronize()
        rows = prog.new_rows()
        assert torch.equal(rows[0], prog.q_idx)
        for b in range(3):  # index keys at their positions
            for j in (0, count[b] - 1) if count[b] else ():
                at = ref[0].at(b, int(first[b]) + j)
                assert torch.equal(prog.k_idx[at], rows[1][b, j])
        for c, x in zip(ref, rows[2:]):
            x = inputs.f32_from_bf16_bits(B.bits_from_bf16(x)).astype(np.float64)
            for b in range(3):
                if count[b]:
                    c.append(b, int(first[b]), x[b, :count[b]])
        for c, b8, sc in ((ref[0], prog.k8, prog.ks), (ref[1], prog.v8, prog.vs)):
            assert C.same_bytes(b8.cpu().numpy(), c.bytes) and np.array_equal(sc.cpu().numpy(), c.scale)
        ki = inputs.f32_from_bf16_bits(B.bits_from_bf16(prog.k_idx)).astype(np.float64)
        qi = inputs.f32_from_bf16_bits(B.bits_from_bf16(prog.q_idx)).astype(np.float64)
        valid = np.minimum(prog.at[:, None], np.maximum(pos + 1, 0))
        mv = []
        for b in range(3):
            rows = np.stack([ki[ref[0].at(b, j)].reshape(-1) for j in range(256)])
            mv.append(C.bf16(rows.reshape(-1, block, 256).sum(1) / block)[0])
        got = prog.idx.cpu().numpy(), prog.n_sel.cpu().numpy()
        _check(prog.sh, block, qi, mv, valid, got)
        sets = [[got[0][b, t, :got[1][b, t]] for t in range(prog.n_q)] for b in range(3)]
        scale = np.float32(prog.sh.softmax_scale)
        for l in range(prog.layers):
            qv = inputs.f32_from_bf16_bits(B.bits_from_bf16(prog.q[l])).astype(np.float64)
            C.check_attention(B.bits_from_bf16(prog.out[l]), prog.lse[l].cpu().numpy().astype(np.float64),
                              C.attention(qv, *ref, sets, scale))
            if l == 0:
                every = [[np.arange(valid[b, t]) for t in range(prog.n_q)] for b in range(3)]
                C.check_attention(B.bits_from_bf16(prog.dense), prog.dense_lse.cpu().numpy().astype(np.float64),
                                  C.attention(qv, *ref, every, scale))


@pytest.mark.parametrize("n_q", [1, 50])
def test_captured_steps(n_q):
    """The path captured into a graph: every replay, with other inputs, gives what eager calls give."""
    import torch
    a, b = (Serving(9, 2, n_q, 512, 32, 128, 64) for _ in range(2))
    for s in (a, b):  # warm up, and allocate what step() allocates
        s.feed([n_q, n_q])
        s.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for _ in range(4):
        for s in (a, b):
            s.feed([n_q, n_q])
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for x, y in zip(a.results(), b.results()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_two_streams_at_once():
    """Two programs on two streams, each with its own buffers, against the same one after another."""
    import torch
    progs = [Serving(s, 2, 40, 512, 64, 128, 0) for s in (1, 2, 1, 2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for p in progs:
            p.feed([40, 13])
        torch.cuda.synchronize()
        for p, st in zip(progs[:2], streams):
            with torch.cuda.stream(st):
                p.step()
        torch.cuda.synchronize()
        for p in progs[2:]:
            p.step()
        torch.cuda.synchronize()
        for i in range(2):
            for x, y in zip(progs[i].results(), progs[i + 2].results()):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_workspace_contents_do_not_matter():
    import torch
    a, b = (Serving(5, 2, 20, 2048, 16, 64, 0) for _ in range(2))
    for _ in range(3):
        for s, fill in ((a, 0), (b, 0xff)):
            for w in s.ws:
                if w is not None:
                    w.fill_(fill)
            s.feed([20, 20])
            s.step()
        torch.cuda.synchronize()
        for x, y in zip(a.results(), b.results()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def _small(key_exp, query_exp):
    """Equal exact scores that fp32 sums tell apart (the order of large and small terms differs),
    of keys and queries whose squares fp32 cannot hold."""
    def tweak(g, qv, mv, blk):
        v = g.integers(-255, 256, size=256) * 2.0 ** g.integers(0, 15, size=256)
        mv[:] = np.stack([g.permutation(v) for _ in range(len(mv))]) * 2.0 ** key_exp
        qv[:] = 2.0 ** query_exp
    return tweak


@pytest.mark.parametrize("key_exp,query_exp", [(0, 0), (-88, 0), (-96, 0), (-104, 0), (0, -70), (0, -90),
                                               (-88, 60), (-50, -52)])
@pytest.mark.parametrize("n_q", [1, 40])
def test_ties_of_small_scores(key_exp, query_exp, n_q):
    _case(n_q, (6400, 3000), 32, 640, 0, n_q, n_q > 1, _small(key_exp, query_exp))


def test_captured_choice_of_many_blocks():
    """The largest form, captured first and replayed between eager calls with other inputs."""
    import torch
    from paper_2606_06467_amd import binding as B
    g = torch.Generator(device="cuda").manual_seed(3)
    sh = _shape(2, 1, 262144, 512)
    lens = torch.tensor([262144, 150001], dtype=torch.int32, device="cuda")
    means = torch.zeros((2, 16384, 256), dtype=torch.bfloat16, device="cuda")
    sides = []
    for _ in "ge":
        sides.append((torch.zeros((2, 1, 256), dtype=torch.bfloat16, device="cuda"), means, None, lens, None,
                      torch.zeros((2, 1, 512), dtype=torch.int32, device="cuda"),
                      torch.zeros((2, 1), dtype=torch.int32, device="cuda"),
                      B.workspace(sh, B.CLSA_OP_BLOCK_TOPK, 16)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.clsa_block_topk(sh, 16, *sides[0])
    for _ in range(4):
        means.copy_(torch.randn(means.shape, generator=g, device="cuda") / 64)
        for s in sides:
            s[0].copy_(torch.randn(s[0].shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda"))
        graph.replay()
        B.clsa_block_topk(sh, 16, *sides[1])
        torch.cuda.synchronize()
        for a, b in zip(sides[0][5:7], sides[1][5:7]):
            assert torch.equal(a, b)
        z = (means.double() @ sides[0][0].double().transpose(1, 2)).squeeze(-1)
        for b, n in enumerate(lens.tolist()):
            own = (n - 1) // 16
            best = set(torch.topk(z[b, :own], 31).indices.tolist()) | {own}
            want = sorted(c * 16 + i for c in best for i in range(16) if c * 16 + i < n)
            assert sides[0][5][b, 0, :len(want)].tolist() == want and int(sides[0][6][b, 0]) == len(want)
