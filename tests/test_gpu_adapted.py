"""Projections with an adapter of each request on the GPU against the formula in 64 bits.

Bounds: sums of n fp32 products, at most gamma_n = n u / (1 - n u) times the sum of magnitudes
(doubled, as for the projections without adapters); the inner sum's two bf16 hold it to 2^-15;
one rounding to bf16, 2^-8."""
import numpy as np
import pytest

from paper_2606_06467_amd import inputs
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def gamma(n):
    return n * U.U32 / (1 - n * U.U32)


def f64(bits):
    return inputs.f32_from_bf16_bits(bits).astype(np.float64)


class Case:
    """Inputs, the cache that they are written to, and the result in 64 bits."""

    def __init__(self, batch, n_q, d, rank, n_adapters, ids, heads=2, page=0, max_len=128, seed=1):
        self.batch, self.n_q, self.d, self.rank, self.heads, self.page, self.max_len = batch, n_q, d, rank, heads, page, max_len
        self.kvw = heads * 128
        self.feats = 512 + 2 * self.kvw
        rng = np.random.default_rng(seed)
        self.h = inputs.normal_bf16(seed, (batch * n_q, d), 1.0)
        self.w = inputs.normal_bf16(seed + 1, (self.feats, d), 0.02)
        self.a = inputs.normal_bf16(seed + 2, (n_adapters, rank, d), 0.05)
        self.b = inputs.normal_bf16(seed + 3, (n_adapters, self.feats, rank), 0.3)
        self.alpha = (rng.random(n_adapters) * 3 - 1).astype(np.float32)
        self.ids = np.asarray(ids, np.int32)
        self.start = rng.integers(0, max_len - n_q + 1, batch).astype(np.int32)
        self.pos = self.start[:, None] + np.arange(n_q, dtype=np.int32)
        self.pos[rng.random(self.pos.shape) < 0.05] = -1
        self.table = None
        if page:
            cols = max_len // page
            self.table = rng.permutation(batch * cols).reshape(batch, cols).astype(np.int32)

    def shape(self):
        from paper_2606_06467_amd import binding as B
        return B.make_shape(self.batch, self.n_q, self.max_len, 1, q_heads=self.heads, kv_heads=self.heads,
                            page_size=self.page, max_pages=self.max_len // self.page if self.page else 0)

    def dev(self):
        import torch
        from paper_2606_06467_amd import binding as B
        bf = {k: B.bf16_from_bits(getattr(self, k)) for k in ("h", "w", "a", "b")}
        it = {k: torch.from_numpy(np.ascontiguousarray(getattr(self, k))).cuda() for k in ("alpha", "ids", "start", "pos")}
        it["table"] = None if self.table is None else torch.from_numpy(self.table).cuda()
        return {**bf, **it}

    def caches(self):
        import torch
        n = self.batch * self.max_len
        return (torch.full((self.batch * self.n_q, 256), 3.0, dtype=torch.bfloat16, device="cuda"),
                *[torch.full((n, k), 3.0, dtype=torch.bfloat16, device="cuda") for k in (256, self.kvw, self.kvw)])

    def run(self, d=None, ws=None):
        from paper_2606_06467_amd import binding as B
        import torch
        d, out = d or self.dev(), self.caches()
        ws = B.workspace(self.shape(), B.CLSA_OP_ADAPTED, self.rank) if ws is None else ws
        ws.fill_(0xFF)   # NaN
        B.clsa_project_append_adapted(self.shape(), self.d, d["h"], d["w"], d["a"], d["b"], d["alpha"], d["ids"],
                                      d["pos"], d["table"], *out, ws)
        torch.cuda.synchronize()
        return [B.bits_from_bf16(t) for t in out]

    def rows(self):
        """Cache row of every token, -1 for none."""
        p = self.pos
        if self.page:
            at = self.table[np.arange(self.batch)[:, None], np.maximum(p, 0) // self.page].astype(np.int64) * self.page + p % self.page
        else:
            at = np.arange(self.batch)[:, None] * self.max_len + p
        return np.where(p >= 0, at, -1).reshape(-1)

    def reference(self):
        h, w = f64(self.h), f64(self.w)
        ref, tol = h @ w.T, 2 * gamma(self.d) * (np.abs(h) @ np.abs(w).T)
        for b, m in enumerate(self.ids):
            if not 0 <= m < len(self.a):
                continue
            r = slice(b * self.n_q, (b + 1) * self.n_q)
            a, up, al = f64(self.a[m]), f64(self.b[m]), float(self.alpha[m])
            ref[r] += al * (h[r] @ a.T) @ up.T
            tol[r] += abs(al) * (2 * gamma(self.d) + 2 * gamma(2 * self.rank) + 2.0 ** -15) * (np.abs(h[r]) @ np.abs(a).T) @ np.abs(up).T
        return ref, tol + np.abs(ref) * 2.0 ** -8 + 1e-30

    def check(self, got, only=None):
        ref, tol = self.reference()
        rows, kvw = self.rows(), self.kvw
        keep = np.ones(len(ref), bool) if only is None else np.repeat(only, self.n_q)
        err = np.abs(f64(got[0][keep]) - ref[keep, :256])
        assert np.all(err <= tol[keep, :256]), float((err / tol[keep, :256]).max())
        for x, c0, c1 in ((got[1], 256, 512), (got[2], 512, 512 + kvw), (got[3], 512 + kvw, 512 + 2 * kvw)):
            live = (rows >= 0) & keep
            err = np.abs(f64(x[rows[live]]) - ref[live, c0:c1])
            assert np.all(err <= tol[live, c0:c1]), float((err / tol[live, c0:c1]).max())
            idle = np.ones(len(x), bool)
            idle[rows[rows >= 0]] = False
            assert np.all(x[idle] == 0x4040)  # 3.0: left as it was


CASES = [  # batch, n_q, d_model, rank, adapters, page
    (1, 1, 512, 8, 1, 0), (5, 1, 2560, 16, 3, 16), (32, 1, 2560, 16, 40, 16), (33, 1, 1024, 64, 5, 0), (70, 1, 4096, 8, 9, 16),
    (128, 1, 512, 128, 130, 0), (200, 1, 512, 16, 11, 16), (3, 5, 1536, 24, 2, 0), (300, 2, 512, 40, 250, 0),
    (7, 37, 512, 16, 3, 16), (1, 300, 2560, 16, 2, 0), (9, 33, 1024, 128, 9, 16), (2, 100, 512, 8, 2, 0), (4, 64, 3584, 56, 3, 0),
    # each form of the tiled product: 64- and 128-row tiles of one sequence and shared ones, by four and eight waves
    (1, 1500, 512, 24, 2, 16), (1500, 1, 512, 40, 50, 0), (250, 5, 512, 128, 9, 16), (1, 2100, 512, 24, 2, 16), (1, 4200, 512, 16, 2, 0), (1, 8300, 512, 40, 1, 16), (2100, 1, 512, 8, 7, 0),
    (700, 6, 512, 24, 60, 16), (30, 150, 512, 72, 4, 16)]


@pytest.mark.parametrize("batch,n_q,d,rank,n,page", CASES)
def test_adapted(batch, n_q, d, rank, n, page):
    rng = np.random.default_rng(batch + n_q)
    ids = rng.integers(-1, n, batch)
    if batch > 2:
        ids[1], ids[2] = -1, n - 1
    max_len = -(-max(n_q + 20, 48) // 16) * 16
    c = Case(batch, n_q, d, rank, n, ids, page=page, max_len=max_len, seed=batch * 7 + rank)
    got = c.run()
    c.check(got)
    for a, b in zip(got, c.run()):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("batch,n_q", [(3, 1), (9, 40)])
def test_adapters_past_32_bits(batch, n_q):
    """The last of adapters that together are larger than 4 GiB."""
    import torch
    rank, n = 128, 18000
    c = Case(batch, n_q, 1024, rank, 3, np.full(batch, 2), max_len=96, seed=11)  # 256 KiB each of A and B
    d = c.dev()
    for k in ("a", "b"):
        t = d[k]
        big = torch.zeros((n, *t.shape[1:]), dtype=t.dtype, device="cuda")
        assert big.nbytes > 1 << 32
        big[-1] = t[2]
        d[k] = big
    d["alpha"] = torch.zeros(n, device="cuda")
    d["alpha"][-1] = float(c.alpha[2])
    d["ids"] = torch.full((batch,), n - 1, dtype=torch.int32, device="cuda")
    c.check(c.run(d))


@pytest.mark.parametrize("batch,n_q", [(6, 1), (150, 1), (3, 70)])
def test_no_adapters_are_the_plain_projections(batch, n_q):
    import torch
    from paper_2606_06467_amd import binding as B
    c = Case(batch, n_q, 1024, 16, 2, np.full(batch, -1), page=16, max_len=96, seed=5)
    d, out = c.dev(), c.caches()
    B.clsa_project_append(c.shape(), c.d, d["h"], d["w"], d["pos"], d["table"], *out)
    torch.cuda.synchronize()
    for a, b in zip(c.run(), out):
        assert np.array_equal(a, B.bits_from_bf16(b))


@pytest.mark.parametrize("batch,n_q", [(6, 1), (150, 1), (5, 70)])
def test_infinities_stay_with_their_adapter(batch, n_q):
    c = Case(batch, n_q, 512, 16, 3, np.arange(batch) % 3 - 1, max_len=96, seed=6)
    c.b[0, :, 3] = 0x7F80      # an infinity against every feature
    c.b[0, 5, 2] = 0x7FC0      # a NaN
    got = c.run()
    others = c.ids != 0
    c.check(got, others)
    q = f64(got[0]).reshape(batch, n_q, 256)
    assert not np.isfinite(q[~others]).any() and np.isnan(q[~others][..., 5]).all()
    # an inner sum that is infinite gives infinities of its features' signs, or NaN where B is zero
    c = Case(batch, n_q, 512, 16, 3, np.arange(batch) % 3 - 1, max_len=96, seed=6)
    c.h[:] = 0x3F80            # ones
    c.a[0, 2] = 0x7F00         # 1.7e38 each: the sum overflows
    c.b[0, 7, 2] = 0
    got = c.run()
    c.check(got, others)
    q = f64(got[0]).reshape(batch, n_q, 256)
    bad = q[~others]
    with np.errstate(invalid="ignore"):
        want = np.sign(f64(c.b[0, :256, 2])) * np.sign(c.alpha[0]) * np.inf
    assert np.isnan(bad[..., 7]).all()
    fine = (np.arange(256) != 7) & np.isinf(want)
    assert fine.sum() > 200
    assert np.array_equal(bad[..., fine], np.broadcast_to(want[fine], bad[..., fine].shape))


@pytest.mark.parametrize("batch,n_q,rank", [(6, 1, 72), (128, 1, 64), (150, 1, 72), (150, 1, 128), (40, 7, 64)])
def test_infinities_among_many_ranks(batch, n_q, rank):
    """Ranks of a feature in lines of their own, and the last of them at an odd place."""
    c = Case(batch, n_q, 512, rank, 3, np.arange(batch) % 3 - 1, max_len=96, seed=8)
    c.b[0, 9, rank - 1] = 0x7F80      # an infinity against one feature
    c.b[0, 14, rank - 8] = 0x7FC0     # a NaN
    got = c.run()
    others = c.ids != 0
    c.check(got, others)
    q = f64(got[0]).reshape(batch, n_q, 256)[~others]
    assert not np.isfinite(q[..., [9, 14]]).any() and np.isnan(q[..., 14]).all()
    assert np.isfinite(np.delete(q, [9, 14], -1)).all()


@pytest.mark.parametrize("batch,n_q", [(6, 1), (150, 1), (5, 70)])
def test_adapter_numbers_out_of_range(batch, n_q):
    from paper_2606_06467_amd import binding as B
    ids = np.arange(batch) % 4
    ids[1], ids[2], ids[3] = 4, -2, 2 ** 31 - 1
    c = Case(batch, n_q, 512, 8, 4, ids, max_len=96, seed=7)
    B.clsa_get_device_error()
    got = c.run()
    assert B.clsa_get_device_error() == B.CLSA_DEVERR_ADAPTER
    c.check(got)


@pytest.mark.parametrize("batch,n_q,rank,block,page", [(4, 1, 16, 16, 0), (140, 1, 8, 16, 16), (5, 77, 64, 32, 64),
                                                       (1, 200, 16, 64, 0)])
def test_adapted_into_the_8bit_cache(batch, n_q, rank, block, page):
    """The same bytes as the rows of the bf16 call, appended."""
    import torch
    from paper_2606_06467_amd import binding as B
    rng = np.random.default_rng(batch)
    max_len = -(-(n_q + 40) // 64) * 64
    c = Case(batch, n_q, 1024, rank, 6, rng.integers(-1, 6, batch), page=page, max_len=max_len, seed=9)
    count = rng.integers(0, n_q + 1, batch).astype(np.int32)
    count[0] = n_q
    c.pos = np.where(np.arange(n_q) < count[:, None], c.start[:, None] + np.arange(n_q), -1).astype(np.int32)
    sh, d, out = c.shape(), c.dev(), c.caches()
    d["count"] = torch.from_numpy(count).cuda()
    ws = B.workspace(sh, B.CLSA_OP_ADAPTED, rank)
    lora = d["a"], d["b"], d["alpha"], d["ids"]
    B.clsa_project_append_adapted(sh, c.d, d["h"], d["w"], *lora, d["pos"], d["table"], *out, ws)
    # rows of K and V in the order of h, from the cache
    rows = torch.from_numpy(np.maximum(c.rows(), 0)).cuda()
    k, v = (out[i][rows].contiguous() for i in (2, 3))

    def cache():
        n = batch * max_len
        return [torch.full((n, c.kvw), 0x20, dtype=torch.uint8, device="cuda") for _ in "kv"] + \
               [torch.full((n // block if page else batch * -(-max_len // block), c.heads), 0.25, device="cuda") for _ in "kv"]

    want, got = cache(), cache()
    B.clsa_cache_append8(sh, block, k, v, d["start"], d["count"], d["table"], *want)
    q, ki = torch.zeros_like(out[0]), torch.full_like(out[1], 3.0)
    ws8 = B.workspace(sh, B.CLSA_OP_ADAPTED8, rank)
    ws8.fill_(0xFF)
    B.clsa_project_append8_adapted(sh, block, c.d, d["h"], d["w"], *lora, d["start"], d["count"], d["table"], q, ki, *got,
                                   ws8)
    torch.cuda.synchronize()
    assert torch.equal(q.view(torch.int16), out[0].view(torch.int16))
    assert torch.equal(ki.view(torch.int16), out[1].view(torch.int16))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("batch,n_q", [(12, 1), (3, 90)])
def test_adapted_replayed(batch, n_q):
    import torch
    from paper_2606_06467_amd import binding as B
    c = Case(batch, n_q, 1024, 16, 4, np.arange(batch) % 5 - 1, max_len=96, seed=3)
    want = c.run()
    d, out, sh = c.dev(), c.caches(), c.shape()
    ws = B.workspace(sh, B.CLSA_OP_ADAPTED, c.rank)

    def step():
        B.clsa_project_append_adapted(sh, c.d, d["h"], d["w"], d["a"], d["b"], d["alpha"], d["ids"], d["pos"],
                                      d["table"], *out, ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for t in out:
            t.fill_(3.0)
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(B.bits_from_bf16(t), w) for t, w in zip(out, want))
        step()
        torch.cuda.synchronize()


def _exact_case(batch, n_q, rank):
    """h = 1, 1, 1, 0 ... and weights -1, -2^-8 in every feature's first two dimensions."""
    c = Case(batch, n_q, 512, rank, 3, np.arange(batch) % 4 - 1, max_len=-(-max(n_q + 8, 48) // 16) * 16, seed=12)
    c.h[:] = 0
    c.h[:, :3] = 0x3F80
    c.w[:] = 0
    c.w[:, 0], c.w[:, 1] = 0xBF80, 0xBB80
    c.a[:], c.b[:] = 0, 0
    c.alpha[:] = 1
    if batch == 1:
        c.ids[:] = 2
    return c


@pytest.mark.parametrize("batch,n_q", [(6, 1), (128, 1), (150, 1), (1500, 1), (2100, 1), (700, 6), (1, 200), (3, 90), (1, 1500), (1, 4200)])
@pytest.mark.parametrize("rank", [8, 24, 64, 72, 128])
def test_inner_sums_keep_24_bits(batch, n_q, rank):
    """u_j = 1 + 2^-8 + 2^-(17 + j mod 7), every product and sum a multiple of 2^-23 below 2: exact in
    fp32 in any order.  Feature f takes rank f mod rank alone, and the weights take 1 + 2^-8 away."""
    c = _exact_case(batch, n_q, rank)
    j = np.arange(rank)
    c.a[:, :, 0], c.a[:, :, 1] = 0x3F80, 0x3B80
    c.a[:, :, 2] = (127 - 17 - j % 7) << 7
    f = np.arange(c.feats)
    c.b[:, f, f % rank] = 0x3F80
    got = c.run()
    want = ((127 - 17 - f % rank % 7) << 7).astype(np.uint16)
    rows, has = c.rows(), np.repeat(c.ids >= 0, n_q)
    for x, c0, at in ((got[0], 0, np.arange(len(rows))), (got[1], 256, rows), (got[2], 512, rows), (got[3], 512 + c.kvw, rows)):
        assert np.array_equal(x[at[(at >= 0) & has]], np.broadcast_to(want[c0:c0 + x.shape[1]], (((at >= 0) & has).sum(), x.shape[1])))
        assert np.all(x[at[(at >= 0) & ~has]] == 0xBF80)   # -(1 + 2^-8): a tie, to the even -1


@pytest.mark.parametrize("batch,n_q", [(6, 1), (150, 1), (1500, 1), (700, 6), (1, 200), (3, 90), (1, 4200)])
@pytest.mark.parametrize("rank", [8, 40, 72, 128])
def test_infinite_upper_factors_keep_their_sign(batch, n_q, rank):
    """u B of a u that is a power of two, any other bf16, an infinity or zero, and an infinite B: the
    product's sign, or NaN for zero."""
    c = _exact_case(batch, n_q, rank)
    c.a[:, :, 0] = np.resize(np.array([0x3F80, 0xBF80, 0x3FC1, 0x0D80, 0x7F7F, 0x7F80, 0xFF80, 0], np.uint16), rank)
    f = np.arange(c.feats)
    j = f % rank
    c.b[:, f, j] = np.where(f // rank % 2, 0xFF80, 0x7F80)
    # the other ranks of a feature are zeros: against an infinite u they would be NaN
    wild = np.flatnonzero(~np.isfinite(f64(c.a[0, :, 0])))
    c.a[:, wild, 0] = 0
    q = f64(c.run()[0])
    u = f64(c.a[0, :, 0])[j[:256]]
    with np.errstate(invalid="ignore"):
        want = u * f64(c.b[0, f, j])[:256]
    has = np.repeat(c.ids >= 0, n_q)
    assert np.array_equal(q[has], np.broadcast_to(want, (has.sum(), 256)), equal_nan=True)
    assert np.all(q[~has] == -1)
    # an infinite u in one rank alone: infinities of both signs of B, and NaN against zeros
    for k in wild[:2]:
        c.a[:, :, 0] = 0
        c.a[:, k, 0] = 0x7F80 if k % 2 else 0xFF80
        c.b[:] = 0
        c.b[:, f, k] = np.resize(np.array([0x3F80, 0xC000, 0x7F80, 0xFF80, 0, 0x0080], np.uint16), c.feats)
        q = f64(c.run()[0])
        with np.errstate(invalid="ignore"):
            want = f64(c.a[0, k:k + 1, 0]) * f64(c.b[0, :256, k])
        assert np.array_equal(q[has], np.broadcast_to(want, (has.sum(), 256)), equal_nan=True)


@pytest.mark.parametrize("batch,n_q", [(6, 1), (128, 1), (150, 1), (1500, 1), (700, 6), (1, 200), (5, 70), (1, 4200)])
@pytest.mark.parametrize("bits", [0x7FFFFFFF, 0xFFFFFFFF, 0x7FFF8000, 0x7F800001, 0x7FC00000])
def test_a_factor_that_is_no_number(batch, n_q, bits):
    """NaN of every payload in alpha: NaN in its sequences' features, and there alone."""
    c = Case(batch, n_q, 512, 16, 3, np.arange(batch) % 4 - 1, max_len=-(-max(n_q + 8, 48) // 16) * 16, seed=13)
    if batch == 1:
        c.ids[:] = 1
    c.alpha[1] = np.array([bits], np.uint32).view(np.float32)[0]
    got = c.run()
    others = c.ids != 1
    c.check(got, others)
    rows, bad = c.rows(), np.repeat(~others, n_q)
    assert np.isnan(f64(got[0][bad])).all()
    for x in got[1:]:
        assert np.isnan(f64(x[rows[bad & (rows >= 0)]])).all()


def test_too_many_tiles_enqueue_nothing():
    """17 million rows of 16896 features are more workgroups than a launch has: refused, and the
    inner sums' place in the workspace is as it was."""
    import torch
    from paper_2606_06467_amd import binding as B
    rows, d, heads = 17_000_000, 512, 64
    sh = B.make_shape(1, rows, 16, 1, q_heads=heads, kv_heads=heads)
    h = torch.ones((rows, d), dtype=torch.bfloat16, device="cuda")
    w, a, b = (torch.ones(s, dtype=torch.bfloat16, device="cuda") for s in ((16896, d), (1, 8, d), (1, 16896, 8)))
    pos, out = torch.full((rows,), -1, dtype=torch.int32, device="cuda"), torch.zeros((rows, 256), dtype=torch.bfloat16, device="cuda")
    ws = B.workspace(sh, B.CLSA_OP_ADAPTED, 8).fill_(0xFF)
    with pytest.raises(B.ClsaError):
        B.clsa_project_append_adapted(sh, d, h, w, a, b, torch.ones(1, device="cuda"),
                                      torch.zeros(1, dtype=torch.int32, device="cuda"), pos, None, out, out, out, out, ws)
    torch.cuda.synchronize()
    kept = bool((ws == 0xFF).all())   # (not in the assertion, which would take the tensor apart)
    assert kept
