"""The operators of the 8-bit shared cache and of block routing, their plain forms and timed cases.

* ``append``: new tokens' K and V into a cache of e4m3 bytes with one power-of-two scale
  for each block of tokens and KV head;
* ``sparse``: attention of a layer's queries over the tokens of an index list, from that cache;
* ``dense``: attention over every valid key of that cache;
* ``route``: the mean index key of each block that new tokens complete, and for every query row
  the tokens of its own block and of the blocks that score best against its index query.

Where ``own`` is false, ``run`` computes an operator from elementary torch operations; where it
is true, it calls the library through its binding."""
import math
import random

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
E4M3 = torch.float8_e4m3fn
D, IDX = 128, 256    # head dimension, index width
E_MIN = -100         # least exponent of a scale
TOP = 240 * 2.0 ** 120  # larger magnitudes are held as this one (its rounding stays finite)


def _case(kind, batch, len_lo, len_hi, **kw):
    c = dict(kind=kind, batch=batch, n_q=1, len_lo=len_lo, len_hi=len_hi, top_k=2048,
             q_heads=32, kv_heads=8, page_size=0, block=64, causal=False)
    c.update(kw)
    return c


def listed():
    return [
        # the new token of every sequence of a serving batch: one row into a block that mostly has some
        dict(_case("append", 32, 1500, 2048, page_size=64), name="append_decode"),
        # a prompt chunk behind half a cache, starting inside a block
        dict(_case("append", 1, 16300, 16300, n_q=8192), name="append_chunk"),
        # a layer of one short conversation: latency is all there is
        dict(_case("sparse", 1, 4096, 4096, top_k=512), name="sparse_4k"),
        # a layer of a small batch of long contexts
        dict(_case("sparse", 4, 131072, 131072), name="sparse_128k"),
        # a layer of a ragged serving batch, paged, smaller blocks than pages
        dict(_case("sparse", 32, 16384, 65536, page_size=64, block=32), name="sparse_paged"),
        # a layer of a prompt chunk whose rows each have an index list of their own (20 / 4 heads)
        dict(_case("sparse", 1, 65536, 65536, n_q=1024, causal=True, q_heads=20, kv_heads=4),
             name="sparse_chunk"),
        # dense attention of a short odd-sized batch: single tokens
        dict(_case("dense", 3, 333, 1001, q_heads=20, kv_heads=4, block=16), name="dense_short"),
        # dense attention of a decode batch: every byte of the cache once
        dict(_case("dense", 8, 32768, 32768), name="dense_decode"),
        # a whole prompt of one cross-decoder layer, causal
        dict(_case("dense", 1, 8192, 8192, n_q=8192, causal=True, q_heads=20, kv_heads=4),
             name="dense_prompt"),
        # block routing of a decode step over long contexts
        dict(_case("route", 4, 131072, 131072), name="route_128k"),
        # the same of a ragged paged batch, two blocks a page
        dict(_case("route", 32, 16384, 65536, page_size=64, block=32, top_k=1024), name="route_paged"),
        # a prompt chunk behind a long context: its blocks' means, and a list for each of its rows
        dict(_case("route", 1, 131072, 131072, n_q=4096, causal=True), name="route_chunk"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same kinds and ranges."""
    qh, kvh = rng.choice([(32, 8), (32, 8), (20, 4), (64, 8), (8, 8), (16, 8)])
    page = rng.choice([0, 64, 128])
    block = rng.choice([16, 32, 64, 64, 128])
    if page:
        block = min(block, page)
    kw = dict(q_heads=qh, kv_heads=kvh, page_size=page, block=block)
    what = rng.choice(["append_decode", "append_chunk", "sparse", "sparse", "sparse_chunk",
                       "dense", "dense_prompt", "route", "route_chunk"])
    if what == "append_decode":
        hi = _log(rng, 200, 4096)
        return _case("append", rng.randint(1, 64), rng.randint(max(8, hi // 2), hi), hi,
                     n_q=rng.choice([1, 1, rng.randint(2, 8)]), **kw)
    if what == "append_chunk":
        batch = rng.randint(1, 3)
        t = _log(rng, 50, 8192 // batch)
        hi = t + _log(rng, 1, 8192)
        return _case("append", batch, max(t, hi - rng.randint(0, 500)), hi, n_q=t, **kw)
    if what == "sparse":
        batch = _log(rng, 1, 32)
        hi = _log(rng, 1000, min(131072, 1500000 // batch))
        k = rng.choice([512, 1024, 2048, rng.randint(1, 2048)])
        return _case("sparse", batch, rng.randint(max(1, hi // 4), hi), hi, top_k=k, **kw)
    if what == "sparse_chunk":
        t = _log(rng, 32, 1024)
        n = _log(rng, 2 * t, 65536)
        k = min(rng.choice([512, 1024, 2048, rng.randint(100, 2048)]), 1024 * 2048 * 4 // (t * kvh))
        return _case("sparse", 1, n, n, n_q=t, causal=True, top_k=k, **kw)
    if what == "dense":
        batch = _log(rng, 1, 32)
        hi = _log(rng, 100, min(131072, 260000 // batch))
        return _case("dense", batch, rng.randint(max(1, hi // 4), hi), hi, **kw)
    if what == "dense_prompt":
        batch = rng.randint(1, 3)
        t = _log(rng, 100, int(8192 / math.sqrt(batch * qh / 20)) if qh > 20 else 8192 // batch)
        return _case("dense", batch, rng.randint(max(1, t // 2), t), t, n_q=t, causal=True, **kw)
    k = block * rng.randint(2, min(2048 // block, 64))
    if what == "route":
        batch = _log(rng, 1, 32)
        hi = _log(rng, 1000, min(131072, 2000000 // batch))
        return _case("route", batch, rng.randint(max(1, hi // 4), hi), hi, top_k=k, **kw)
    t = _log(rng, 50, 4096)
    n = _log(rng, 2 * t, 131072 if block >= 64 else 2048 * block)
    return _case("route", 1, n, n, n_q=t, causal=True, top_k=k, **kw)


def _lens(c):
    """Cached tokens of each sequence: the longest first, the rest between the two bounds."""
    r = random.Random(c["batch"] * 1000003 + c["len_lo"])
    return [c["len_hi"]] + [r.randint(c["len_lo"], c["len_hi"]) for _ in range(c["batch"] - 1)]


def _max_len(c):
    p = c["page_size"]
    return -(-c["len_hi"] // p) * p if p else c["len_hi"]


def _valid(c):
    """Valid keys of every row, as lists: causal rows are the last n_q of their sequence."""
    t = c["n_q"]
    return [[max(0, n - t + i + 1) if c["causal"] else n for i in range(t)] for n in _lens(c)]


def _rows(c):
    """Shape of a cache's token rows, and of its blocks."""
    p, s = c["page_size"], c["block"]
    if p:
        pages = sum(-(-n // p) for n in _lens(c))
        return (pages, p), (pages, p // s)
    return (c["batch"], _max_len(c)), (c["batch"], -(-_max_len(c) // s))


def _page_table(c, gen):
    p = c["page_size"]
    if not p:
        return None
    need = [-(-n // p) for n in _lens(c)]
    perm = torch.randperm(sum(need), generator=gen, device=DEV).to(I32)
    pt = torch.full((c["batch"], _max_len(c) // p), -1, dtype=I32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        pt[b, :n] = perm[at:at + n]
        at += n
    return pt


def _normal(gen, shape, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEV).mul_(scale).to(BF16)


def _filled(c, gen):
    """A filled 8-bit cache of one of K and V: bytes and scales; channels differ in size."""
    (n0, n1), (m0, m1) = _rows(c)
    h, s = c["kv_heads"], c["block"]
    b8 = torch.zeros((n0, n1, h, D), dtype=U8, device=DEV)
    sc = torch.ones((m0, m1, h), device=DEV)
    size = torch.exp(0.5 * torch.randn((h, D), generator=gen, device=DEV))
    step = max(1, (1 << 17) // n1)
    for i in range(0, n0, step):
        k = min(step, n0 - i)
        x = torch.randn((k, m1 * s, h, D), generator=gen, device=DEV) * size
        x[:, n1:] = 0
        x = x.view(k, m1, s, h, D)
        e = torch.ceil(torch.log2(x.abs().amax((2, 4)) / 448))
        sc[i:i + k] = torch.exp2(e)
        x = x / torch.exp2(e)[:, :, None, :, None]
        b8[i:i + k] = x.to(E4M3).view(U8).reshape(k, m1 * s, h, D)[:, :n1]
    return b8.view(E4M3), sc


def prepare(c, seed):
    """Inputs and output buffers of one case."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kind, bt, t, hq, h = c["kind"], c["batch"], c["n_q"], c["q_heads"], c["kv_heads"]
    lens = _lens(c)
    rows, blocks = _rows(c)
    s = dict(case=c, page_table=_page_table(c, gen))
    s["seq_lens"] = torch.tensor(lens, dtype=I32, device=DEV)
    s["q_pos"] = None
    if c["causal"]:  # rows before a shorter sequence's first token see nothing
        s["q_pos"] = torch.tensor([[n - t + i for i in range(t)] for n in lens], dtype=I32, device=DEV)
    # the new tokens are the last of their sequence
    new = [min(t, n) for n in lens]
    s["start"] = torch.tensor([n - m for n, m in zip(lens, new)], dtype=I32, device=DEV)
    s["count"] = torch.tensor(new, dtype=I32, device=DEV)
    if kind == "append":
        s["k8"], s["k_scale"] = _filled(c, gen)
        s["v8"], s["v_scale"] = _filled(c, gen)
        # some new tokens are larger than what their block held
        big = torch.exp(torch.randn((bt, t, 1, 1), generator=gen, device=DEV))
        s["k"] = (torch.randn((bt, t, h, D), generator=gen, device=DEV) * big).to(BF16)
        s["v"] = (torch.randn((bt, t, h, D), generator=gen, device=DEV) * big).to(BF16)
    elif kind in ("sparse", "dense"):
        s["k8"], s["k_scale"] = _filled(c, gen)
        s["v8"], s["v_scale"] = _filled(c, gen)
        s["q"] = _normal(gen, (bt, t, hq, D))
        s["out"] = torch.zeros((bt, t, hq, D), dtype=BF16, device=DEV)
        s["lse"] = torch.zeros((bt, t, hq), device=DEV)
    if kind == "sparse":  # ascending lists, one token out of each equal share of the valid ones
        k = c["top_k"]
        n = torch.tensor(_valid(c), device=DEV)[..., None]
        m = n.clamp(max=k)
        i = torch.arange(k, device=DEV)
        lo, hi = i * n // m.clamp(min=1), (i + 1) * n // m.clamp(min=1)
        u = torch.rand((bt, t, k), generator=gen, device=DEV, dtype=F64)
        j = torch.minimum(lo + (u * (hi - lo)).long(), hi - 1)
        s["idx"] = torch.where(i < m, j, -1).to(I32)
        s["n_sel"] = m[..., 0].to(I32)
    if kind == "route":
        s["q_idx"] = _normal(gen, (bt, t, 4, IDX // 4), 1 / 8)
        s["k_idx"] = _normal(gen, rows + (4, IDX // 4), 1 / 8)
        s["means"] = _normal(gen, blocks + (IDX,), 1 / 8 / math.sqrt(c["block"]))
        s["idx"] = torch.full((bt, t, c["top_k"]), -1, dtype=I32, device=DEV)
        s["n_sel"] = torch.zeros((bt, t), dtype=I32, device=DEV)
    return s


def _token_rows(s, b, j):
    """Row of token j of sequence b in a cache seen as [tokens, ...] (j: int64)."""
    c = s["case"]
    p = c["page_size"]
    if not p:
        return b * _max_len(c) + j
    return s["page_table"][b, j // p].long() * p + j % p


def _block_rows(s, b, blk):
    """Row of block blk of sequence b in what is kept for each block."""
    c = s["case"]
    p, n = c["page_size"], c["block"]
    if not p:
        return b * (-(-_max_len(c) // n)) + blk
    return s["page_table"][b, blk * n // p].long() * (p // n) + blk * n % p // n


def _values(s, what, b, j):
    """The cached K or V rows of tokens j of sequences b, in float32."""
    h = s["case"]["kv_heads"]
    x = s[what + "8"].view(U8).view(-1, h, D)[_token_rows(s, b, j)].view(E4M3).to(F32)
    return x * s[what + "_scale"].view(-1, h)[_block_rows(s, b, j // s["case"]["block"])][..., None]


def _touched(s):
    """Blocks that the new tokens reach, [batch, blocks]; a sequence's last one stands for those past it."""
    n = s["case"]["block"]
    start, last = s["start"].long(), (s["start"] + s["count"]).long() - 1
    most = (s["case"]["n_q"] + n - 2) // n + 1
    blk = start[:, None] // n + torch.arange(most, device=DEV)
    return torch.minimum(blk, last[:, None] // n)


def _append(s, what):
    c = s["case"]
    n, h = c["block"], c["kv_heads"]
    blk = _touched(s)                                           # [batch, blocks]
    b = torch.arange(c["batch"], device=DEV)[:, None]
    start, end = s["start"].long()[:, None, None], (s["start"] + s["count"]).long()[:, None, None]
    pos = blk[..., None] * n + torch.arange(n, device=DEV)      # [batch, blocks, n]
    new, kept = (pos >= start) & (pos < end), pos < start
    x = s[what][b[..., None], (pos - start).clamp(0, c["n_q"] - 1)].to(F32).clamp(-TOP, TOP)
    a = torch.where(new[..., None, None], x, 0).abs().amax((2, 4))
    m, e = torch.frexp(a)                                       # 448 = 0.875 * 2^9
    e = torch.where(a > 0, e - 9 + (m > 0.875).to(e.dtype), E_MIN).clamp(min=E_MIN)
    fresh = torch.ldexp(torch.ones_like(a), e)
    scales, at = s[what + "_scale"].view(-1, h), _block_rows(s, b, blk)
    old = scales[at]
    sc = torch.where(kept.any(-1)[..., None], torch.maximum(old, fresh), fresh)
    byte = s[what + "8"].view(U8).view(-1, h, D)
    # the last block of a cache whose length is no multiple of n ends early
    rows = _token_rows(s, b[..., None], pos.clamp(max=_max_len(c) - 1))
    was = byte[rows]
    moved = (was.view(E4M3).to(F32) * (old / sc)[:, :, None, :, None]).to(E4M3).view(U8)
    put = (x / sc[:, :, None, :, None]).to(E4M3).view(U8)
    now = torch.where(new[..., None, None], put, torch.where(kept[..., None, None], moved, was))
    inside = (pos < _max_len(c))[..., None, None]
    last = _token_rows(s, b[..., None], torch.full_like(pos, _max_len(c) - 1))
    if _max_len(c) % n:  # rows past the end repeat the last token's
        i = ((_max_len(c) - 1) % n)
        now = torch.where(inside, now, now[:, :, i:i + 1])
        rows = torch.where(inside[..., 0, 0], rows, last)
    byte[rows] = now
    scales[at] = sc


def _attend(s, k, v, live):
    """Softmax attention of q [batch, rows, heads] over its keys, those where live."""
    c = s["case"]
    h, g = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    bt, t = c["batch"], c["n_q"]
    q = s["q"].to(F32).view(bt, t, h, g, D) * (1 / math.sqrt(D))
    if k.dim() == 5:   # a list per row: [batch, rows, keys, heads, D]
        z = torch.matmul(q, k.permute(0, 1, 3, 4, 2))           # [batch, rows, h, g, keys]
        z = z.masked_fill(~live[:, :, None, None], -math.inf)
    else:              # [batch, keys, heads, D]
        z = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(bt, h, g * t, D), k.permute(0, 2, 3, 1))
        z = z.view(bt, h, g, t, -1).masked_fill(~live[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    z -= torch.where(top == -math.inf, 0, top)
    z.exp_()
    total = z.sum(-1, keepdim=True)
    lse = torch.log(total) + top
    z /= torch.where(total == 0, 1, total)
    if k.dim() == 5:
        o = torch.matmul(z, v.permute(0, 1, 3, 2, 4))
        lse = lse[..., 0]
    else:
        o = torch.matmul(z.view(bt, h, g * t, -1), v.permute(0, 2, 1, 3))
        o, lse = o.view(bt, h, g, t, D).permute(0, 3, 1, 2, 4), lse[..., 0].permute(0, 3, 1, 2)
    return dict(out=o.reshape(bt, t, h * g, D).to(BF16), lse=lse.reshape(bt, t, h * g).contiguous())


def _counts(s):
    """Valid keys of every row, [batch, rows]."""
    n = s["seq_lens"].long()[:, None]
    if s["q_pos"] is None:
        return n.expand(-1, s["case"]["n_q"])
    return torch.minimum(n, (s["q_pos"].long() + 1).clamp(min=0))


def _route(s):
    c = s["case"]
    n, kb = c["block"], c["top_k"] // c["block"]
    bt = c["batch"]
    b = torch.arange(bt, device=DEV)[:, None]
    # means of the blocks that the new tokens complete (sums in 64 bits)
    blk = _touched(s)
    whole = (blk + 1) * n <= (s["start"] + s["count"]).long()[:, None]
    pos = (blk[..., None] * n + torch.arange(n, device=DEV)).clamp(max=_max_len(c) - 1)
    mean = s["k_idx"].view(-1, IDX)[_token_rows(s, b[..., None], pos)].to(F64).mean(2)
    flat, at = s["means"].view(-1, IDX), _block_rows(s, b, blk)
    flat[at] = torch.where(whole[..., None], mean.to(F32).to(BF16), flat[at])
    # scores of the blocks before each row's own, next to a border of the selection: 64 bits
    most = -(-_max_len(c) // n)
    p = c["page_size"]
    blocks = torch.arange(most, device=DEV)
    held = blocks * n // p if p else blocks
    owned = _block_rows(s, b, blocks) if not p else \
        s["page_table"][:, held].long().clamp(min=0) * (p // n) + blocks * n % p // n
    keys = flat[owned].to(F64)                                  # [batch, blocks, 256]
    z = torch.matmul(s["q_idx"].view(bt, c["n_q"], IDX).to(F64), keys.transpose(1, 2))
    valid = _counts(s)[..., None]
    mine = (valid - 1).clamp(min=0) // n
    z = torch.where(blocks == mine, math.inf, torch.where(blocks < mine, z, -math.inf))
    order = torch.sort(z, dim=-1, descending=True, stable=True).indices[..., :kb]
    if most < kb:
        order = torch.cat([order, order.new_full(order.shape[:2] + (kb - most,), most)], -1)
    order = torch.sort(torch.where(order <= mine, order, most + kb), -1).values
    tok = (order[..., None] * n + torch.arange(n, device=DEV)).flatten(2)
    s["idx"] = torch.where(tok < valid, tok, -1).to(I32)
    s["n_sel"] = (tok < valid).sum(-1).to(I32)
    return dict(means=s["means"], idx=s["idx"], n_sel=s["n_sel"])


def _plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "append":
        _append(s, "k")
        _append(s, "v")
        return {k: s[k] for k in ("k8", "v8", "k_scale", "v_scale")}
    if kind == "route":
        return _route(s)
    b = torch.arange(c["batch"], device=DEV)
    if kind == "sparse":
        j = s["idx"].long().clamp(min=0)
        b = b[:, None, None]
        return _attend(s, _values(s, "k", b, j), _values(s, "v", b, j),
                       torch.arange(c["top_k"], device=DEV) < s["n_sel"][..., None])
    j = torch.arange(c["len_hi"], device=DEV)
    held = torch.minimum(j, s["seq_lens"].long()[:, None] - 1)  # keys past the end: the last one's
    b = b[:, None]
    return _attend(s, _values(s, "k", b, held), _values(s, "v", b, held), j < _counts(s)[..., None])


def _handles(s):
    """The shape and workspace that a program keeps beside its buffers."""
    from paper_2606_06467_amd import binding as B
    c = s["case"]
    if "shape" not in s:
        m, p = _max_len(c), c["page_size"]
        s["shape"] = B.make_shape(c["batch"], c["n_q"], m, c["top_k"], q_heads=c["q_heads"],
                                  kv_heads=c["kv_heads"], page_size=p,
                                  max_pages=m // p if p else 0, causal=c["causal"])
        op = dict(sparse="CLSA_OP_ATTN8", dense="CLSA_OP_DENSE8", route="CLSA_OP_BLOCK_TOPK")
        s["ws"] = None
        if c["kind"] in op:
            s["ws"] = B.workspace(s["shape"], getattr(B, op[c["kind"]]), c["block"], DEV)
    return B, s["shape"], c["block"], s["page_table"]


def _library(s):
    kind = s["case"]["kind"]
    B, sh, n, pt = _handles(s)
    if kind == "append":
        B.clsa_cache_append8(sh, n, s["k"], s["v"], s["start"], s["count"], pt, s["k8"], s["v8"],
                             s["k_scale"], s["v_scale"])
        return {k: s[k] for k in ("k8", "v8", "k_scale", "v_scale")}
    if kind == "route":
        B.clsa_block_means(sh, n, s["k_idx"], s["start"], s["count"], pt, s["means"])
        B.clsa_block_topk(sh, n, s["q_idx"], s["means"], pt, s["seq_lens"], s["q_pos"], s["idx"],
                          s["n_sel"], s["ws"])
        return dict(means=s["means"], idx=s["idx"], n_sel=s["n_sel"])
    cache = s["k8"], s["v8"], s["k_scale"], s["v_scale"], pt
    if kind == "sparse":
        B.clsa_sparse_attn8(sh, n, s["q"], *cache, s["idx"], s["n_sel"], s["out"], s["lse"], s["ws"])
    else:
        B.clsa_dense_attn8(sh, n, s["q"], *cache, s["seq_lens"], s["q_pos"], s["out"], s["lse"], s["ws"])
    return dict(out=s["out"], lse=s["lse"])


def run(s):
    return _library(s) if own else _plain(s)


def work(c):
    kind, bt, t, hq, h, n = c["kind"], c["batch"], c["n_q"], c["q_heads"], c["kv_heads"], c["block"]
    lens, valid = _lens(c), _valid(c)
    rows = bt * t
    if kind == "append":
        tok = sum(min(t, m) for m in lens)
        held = sum(len(range((m - min(t, m)) // n, -(-m // n))) for m in lens)  # blocks reached
        return dict(bytes=2 * tok * h * D * 3 + 2 * held * h * 8 + 8 * bt, flops=4 * tok * h * D)
    if kind == "route":
        done = sum(m // n - (m - min(t, m)) // n for m in lens)  # blocks completed
        scored = [sum(max(0, -(-v // n) - 1) for v in vs) for vs in valid]
        seen = sum(max(0, -(-max(vs) // n) - 1) for vs in valid)
        return dict(bytes=done * (n + 1) * 2 * IDX + (seen + rows) * 2 * IDX + rows * (c["top_k"] + 1) * 4,
                    flops=2 * IDX * sum(scored) + done * n * IDX)
    if kind == "sparse":
        keys = [sum(min(v, c["top_k"]) for v in vs) for vs in valid]
        # each cached row and scale once at most, however many lists hold it
        held = sum(min(k, max(vs)) for k, vs in zip(keys, valid))
        more = sum(keys) * 4 + rows * 4
    else:
        keys = [sum(vs) for vs in valid]
        held = sum(max(vs) for vs in valid)
        more = 0
    scales = min(held, sum(-(-m // n) for m in lens)) * h * 8
    return dict(bytes=held * h * 2 * D + scales + rows * hq * (4 * D + 4) + more,
                flops=4 * hq * D * sum(keys))


def _exact_cache(s, what, b):
    """Sequence b's cached rows in 64 bits, as numbers: [tokens, heads, D]."""
    c = s["case"]
    n, p, m = c["block"], c["page_size"], _lens(c)[b]
    x, f = s[what + "8"].to(F32).to(F64), s[what + "_scale"].to(F64)
    if p:
        pages = s["page_table"][b, :-(-m // p)].long()
        x, f = x[pages].flatten(0, 1), f[pages].flatten(0, 1)
    else:
        x, f = x[b], f[b]
    return x[:m] * f.repeat_interleave(n, 0)[:m, :, None]


def _exact_attention(s):
    c = s["case"]
    h, g, t = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["n_q"]
    out = torch.zeros(s["out"].shape, dtype=F64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=F64, device=DEV)
    for b, m in enumerate(_lens(c)):
        k, v = _exact_cache(s, "k", b), _exact_cache(s, "v", b)
        limit = torch.tensor(_valid(c)[b], device=DEV)
        for i in range(0, t, 1024):
            rows = slice(i, min(t, i + 1024))
            for a in range(h):
                q = s["q"][b, rows, a * g:(a + 1) * g].to(F64) / math.sqrt(D)   # [rows, g, D]
                if c["kind"] == "sparse":
                    sel = s["idx"][b, rows].long()
                    kk, vv = k[sel.clamp(min=0), a], v[sel.clamp(min=0), a]     # [rows, keys, D]
                    z = torch.bmm(q, kk.transpose(1, 2).contiguous())
                    z[(sel < 0)[:, None].expand_as(z)] = -math.inf
                else:
                    z = (q.reshape(-1, D) @ k[:, a].T).view(-1, g, m)
                    z.masked_fill_((torch.arange(m, device=DEV) >= limit[rows, None])[:, None], -math.inf)
                lse[b, rows, a * g:(a + 1) * g] = torch.logsumexp(z, -1)
                w = torch.softmax(z, -1).nan_to_num_(0.0)
                o = torch.bmm(w, vv) if c["kind"] == "sparse" else (w.view(-1, m) @ v[:, a]).view(-1, g, D)
                out[b, rows, a * g:(a + 1) * g] = o
    return dict(out=out, lse=lse)


def _exact_append(s):
    """Values over their block's scale, not rounded, and the scales."""
    c = s["case"]
    n, p = c["block"], c["page_size"]
    r = {}
    for what in ("k", "v"):
        x8, f = s[what + "8"].to(F32).to(F64), s[what + "_scale"].to(F64)
        for b, m in enumerate(_lens(c)):
            first = int(s["start"][b])
            for blk in range(first // n, -(-m // n)):
                at, upto = max(first, blk * n), min(m, blk * n + n)
                x = s[what][b, at - first:upto - first].to(F64)          # [tokens, heads, D]
                need = torch.exp2(torch.ceil(torch.log2(x.abs().amax((0, 2)) / 448)))
                if p:
                    page, off = int(s["page_table"][b, blk * n // p]), blk * n % p
                    block, scale = x8[page, off:off + n], f[page]
                    i = off // n
                else:
                    block, scale, i = x8[b, blk * n:blk * n + n], f[b], blk
                have = scale[i].clone()
                scale[i] = torch.maximum(have, need) if at > blk * n else need
                block[:at - blk * n] *= (have / scale[i])[:, None]
                block[at - blk * n:upto - blk * n] = x / scale[i][:, None]
        r[what + "8"], r[what + "_scale"] = x8, f
    return r


def exact(c, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    if c["kind"] == "route":
        # whole numbers, and means that the sums' one rounding decides
        s = prepare(c, seed)
        n, p = c["block"], c["page_size"]
        means = s["means"].to(F64)
        for b, m in enumerate(_lens(c)):
            for blk in range(int(s["start"][b]) // n, m // n):
                if p:
                    page, off = int(s["page_table"][b, blk * n // p]), blk * n % p
                    means[page, off // n] = s["k_idx"][page, off:off + n].to(F64).sum(0).flatten() / n
                else:
                    means[b, blk] = s["k_idx"][b, blk * n:blk * n + n].to(F64).sum(0).flatten() / n
        return dict(means=means, idx=None, n_sel=None)
    if c["kind"] == "append":
        if c["batch"] * c["n_q"] // c["block"] > 4000:
            return None
        return _exact_append(prepare(c, seed))
    return _exact_attention(prepare(c, seed))
