"""A serving step of many requests: the norm, the projections with each request's adapter,
forks and pages, and the decode step over them, as they are used together."""
import numpy as np
import pytest

from paper_2606_06467_amd import inputs

pytestmark = pytest.mark.gpu
D, RANK, PAGE, COLS, SLOTS, L, K = 1024, 16, 64, 8, 6, 2, 128


class Server:
    """SLOTS slots over one pool of pages, in bf16 (with what a step needs)."""

    def __init__(self, pages, seed):
        import torch
        from paper_2606_06467_amd import binding as B
        self.B, self.torch, self.pages = B, torch, pages
        bf = lambda i, s, x: B.bf16_from_bits(inputs.normal_bf16(seed + i, s, x))  # noqa: E731
        feats = 512 + 2 * 8 * 128
        self.w, self.nw = bf(1, (feats, D), 0.03), bf(2, (D,), 1.0)
        self.a, self.b = bf(3, (3, RANK, D), 0.05), bf(4, (3, feats, RANK), 0.2)
        self.alpha = torch.tensor([0.5, 1.0, 2.0], device="cuda")
        z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.cache = [z(pages, PAGE, 4, 64), z(pages, PAGE, 8, 128), z(pages, PAGE, 8, 128)]
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.refs, self.lens, self.missing = i32(SLOTS, COLS) - 1, i32(pages), i32(SLOTS), i32(1)
        self.adapter = torch.tensor([0, 1, -1, 2, 0, 1], dtype=torch.int32, device="cuda")

    def shape(self, n_q):
        return self.B.make_shape(SLOTS, n_q, COLS * PAGE, K, page_size=PAGE, max_pages=COLS, causal=n_q > 1)

    def fork(self, parent):
        p = self.torch.tensor(parent, dtype=self.torch.int32, device="cuda")
        self.B.clsa_pages_fork(self.shape(1), p, self.table, self.lens, self.refs)

    def append(self, x, r, count):
        """New tokens of every slot: the norm, pages, projections.  x, r: [SLOTS, n_q, D]."""
        B, torch, n_q = self.B, self.torch, x.shape[1]
        sh = self.shape(n_q)
        n = torch.tensor(count, dtype=torch.int32, device="cuda")
        s, h = torch.empty_like(x), torch.empty_like(x)
        B.clsa_residual_norm(sh, D, 1e-6, x, r, self.nw, s, h)
        B.clsa_pages_reserve(sh, self.cache, self.lens, n, self.table, self.refs, self.missing,
                             B.workspace(sh, B.CLSA_OP_PAGES_RESERVE))
        t = torch.arange(n_q, device="cuda", dtype=torch.int32)
        pos = torch.where(t < n[:, None], self.lens[:, None] + t, -1)
        q = torch.empty((SLOTS, n_q, 4, 64), dtype=torch.bfloat16, device="cuda")
        B.clsa_project_append_adapted(sh, D, h, self.w, self.a, self.b, self.alpha, self.adapter, pos, self.table,
                                      q, *self.cache, B.workspace(sh, B.CLSA_OP_ADAPTED, RANK))
        self.lens += n
        assert int(self.missing[0]) == 0
        return q

    def decode(self, q, ql):
        B, torch = self.B, self.torch
        sh = self.shape(1)
        out = torch.zeros((L, SLOTS, 1, 32, 128), dtype=torch.bfloat16, device="cuda")
        idx = torch.zeros((SLOTS, 1, K), dtype=torch.int32, device="cuda")
        ns = torch.zeros((SLOTS, 1), dtype=torch.int32, device="cuda")
        B.clsa_decode_step(sh, q, *self.cache, self.table, self.lens, None, ql, out, None, idx, ns,
                           B.workspace(sh, B.CLSA_OP_DECODE, L))
        return out, idx, ns


def _tokens(seed, n_q):
    from paper_2606_06467_amd import binding as B
    return [B.bf16_from_bits(inputs.normal_bf16(seed + i, (SLOTS, n_q, D), 1.0)) for i in range(2)]


def test_forked_requests_like_requests_of_their_own():
    """Two prompts, forked to samples that go on with tokens of their own: the same index sets
    and outputs, bit for bit, as with a pool in which every slot appends its whole text itself;
    the same again after other requests have gone and the pool is compacted."""
    import torch
    from paper_2606_06467_amd import binding as B
    shared, alone = Server(90, 50), Server(90, 50)
    prompt = _tokens(10, 150)
    same = [p.clone() for p in prompt]
    for p in (*prompt, *same):          # the samples' adapters are their prompt's
        p[1:4], p[4:] = p[:1], p[4:5]
    ids = torch.tensor([0, 0, 0, 0, 2, 2], dtype=torch.int32, device="cuda")
    shared.adapter, alone.adapter = ids, ids
    B.clsa_get_device_error()
    shared.append(*prompt, [150, 0, 0, 0, 75, 0])
    shared.fork([0, 0, 0, 0, 4, 4])
    alone.append(*same, [150, 150, 150, 150, 75, 75])
    assert int((shared.refs > 0).sum()) == 5 and int((alone.refs > 0).sum()) == 16
    ql = torch.randn((L, SLOTS, 1, 32, 128), generator=torch.Generator().manual_seed(1)).cuda().to(torch.bfloat16)
    for t in range(3):
        x = _tokens(100 + t, 1)
        got = [s.decode(s.append(*x, [1] * SLOTS), ql) for s in (shared, alone)]
        for a, b in zip(*got):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), t
        # the prompts' whole pages are shared, the last one is each slot's own (one keeps the first)
        assert int((shared.refs > 0).sum()) == 2 + 4 + 1 + 2
    # samples end; what is left moves to the front and decodes as before
    shared.fork([-1, 1, -1, 3, 4, -1])
    alone.fork([-1, 1, -1, 3, 4, -1])
    bound = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.clsa_pages_compact(shared.shape(1), shared.cache, shared.table, shared.refs, bound,
                         B.workspace(shared.shape(1), B.CLSA_OP_PAGES_COMPACT, shared.pages))
    assert int(bound[0]) == int((shared.refs > 0).sum()) == 2 + 2 + 1 + 1
    x = _tokens(300, 1)
    got = [s.decode(s.append(*x, [0, 1, 0, 1, 1, 0]), ql) for s in (shared, alone)]
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(shared.lens, alone.lens) and B.clsa_get_device_error() == 0


@pytest.mark.parametrize("block", [16, 64])
def test_forks_of_the_8bit_cache(block):
    """The same over the 8-bit cache, with its scales and block keys among a page's tensors: dense
    and block-routed attention of forked requests, bit for bit as of requests of their own."""
    import torch
    from paper_2606_06467_amd import binding as B
    gen = torch.Generator().manual_seed(3)
    ids = torch.tensor([0, 0, 0, 0, 2, 2], dtype=torch.int32, device="cuda")
    n = PAGE // block

    def server():
        s = Server(90, 60)
        s.adapter = ids
        u8 = lambda *d: torch.zeros(d, dtype=torch.uint8, device="cuda")  # noqa: E731
        s.k8, s.v8 = u8(90, PAGE, 8, 128), u8(90, PAGE, 8, 128)
        s.ks, s.vs = (torch.ones((90, n, 8), device="cuda") for _ in "kv")
        s.means = torch.zeros((90, n, 256), dtype=torch.bfloat16, device="cuda")
        s.cache = [s.cache[0], s.k8, s.v8, s.ks, s.vs, s.means]
        return s

    def append(s, h, count):
        n_q = h.shape[1]
        sh = s.shape(n_q)
        c = torch.tensor(count, dtype=torch.int32, device="cuda")
        B.clsa_pages_reserve(sh, s.cache, s.lens, c, s.table, s.refs, s.missing, B.workspace(sh, B.CLSA_OP_PAGES_RESERVE))
        q = torch.empty((SLOTS, n_q, 4, 64), dtype=torch.bfloat16, device="cuda")
        B.clsa_project_append8_adapted(sh, block, D, h, s.w, s.a, s.b, s.alpha, s.adapter, s.lens, c, s.table, q,
                                       s.cache[0], s.k8, s.v8, s.ks, s.vs, B.workspace(sh, B.CLSA_OP_ADAPTED8, RANK))
        B.clsa_block_means(sh, block, s.cache[0], s.lens, c, s.table, s.means)
        s.lens += c
        assert int(s.missing[0]) == 0
        return q

    def attend(s, q_idx, q):
        sh = s.shape(1)
        dense, sparse = torch.zeros_like(q), torch.zeros_like(q)
        cache = s.k8, s.v8, s.ks, s.vs, s.table
        B.clsa_dense_attn8(sh, block, q, *cache, s.lens, None, dense, ws=B.workspace(sh, B.CLSA_OP_DENSE8))
        idx = torch.zeros((SLOTS, 1, K), dtype=torch.int32, device="cuda")
        ns = torch.zeros((SLOTS, 1), dtype=torch.int32, device="cuda")
        B.clsa_block_topk(sh, block, q_idx, s.means, s.table, s.lens, None, idx, ns,
                          B.workspace(sh, B.CLSA_OP_BLOCK_TOPK, block))
        B.clsa_sparse_attn8(sh, block, q, *cache, idx, ns, sparse, ws=B.workspace(sh, B.CLSA_OP_ATTN8))
        return dense, sparse, idx, ns

    shared, alone = server(), server()
    prompt = torch.randn((SLOTS, 150, D), generator=gen).cuda().to(torch.bfloat16)
    same = prompt.clone()
    same[1:4], same[4:] = same[:1], same[4:5]
    append(shared, prompt, [150, 0, 0, 0, 75, 0])
    shared.fork([0, 0, 0, 0, 4, 4])
    append(alone, same, [150, 150, 150, 150, 75, 75])
    for t in range(4):
        h = torch.randn((SLOTS, 9, D), generator=gen).cuda().to(torch.bfloat16)
        q = torch.randn((SLOTS, 1, 32, 128), generator=gen).cuda().to(torch.bfloat16)
        count = [9, 8, 7, 1, 0, 9]
        got = []
        for s in (shared, alone):
            qi = append(s, h, count)
            got.append(attend(s, qi[:, :1].contiguous(), q))
        for a, b in zip(*got):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), t
        if t == 2:
            bound = torch.zeros(1, dtype=torch.int32, device="cuda")
            B.clsa_pages_compact(shared.shape(1), shared.cache, shared.table, shared.refs, bound,
                                 B.workspace(shared.shape(1), B.CLSA_OP_PAGES_COMPACT, shared.pages))
            assert int(bound[0]) == int((shared.refs > 0).sum())
