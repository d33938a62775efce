"""Operators around the shared cache of many requests, their plain forms and timed cases.

* ``norm``: the residual's addition and the root-mean-square norm in front of the projections, its
  result as bf16 and as e4m3 bytes with power-of-two scales;
* ``norm_grad``: its backward pass;
* ``adapt``: the projections of new tokens with a low-rank adapter of each request beside the shared
  weights, written into the bf16 or the 8-bit cache;
* ``fork``: slots of a paged cache become forks of others, and get pages to write into (pages that
  they share are copied first);
* ``compact``: the pages in use move to the front of the pool.

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
EPS = 1e-6


def _norm(rows, d, group=0, bf16=True, residual=True):
    """group: values that share a scale of the 8-bit result (d: a whole row), 0 for none."""
    return dict(kind="norm", rows=rows, d=d, group=group, bf16=bf16, residual=residual)


def _grad(rows, d, residual=True):
    return dict(kind="norm_grad", rows=rows, d=d, residual=residual)


def _adapt(batch, n_q, len_hi, **kw):
    c = dict(kind="adapt", batch=batch, n_q=n_q, len_hi=len_hi, d=2560, rank=16, adapters=8, kv_heads=8,
             q_heads=32, page_size=64, bits8=False, block=64, ragged=False)
    c.update(kw)
    return c


def _fork(prompts, samples, len_lo, len_hi, **kw):
    c = dict(kind="fork", prompts=prompts, samples=samples, len_lo=len_lo, len_hi=len_hi, n_q=1,
             page_size=64, kv_heads=8, bits8=False, block=64)
    c.update(kw)
    return c


def _compact(pages, used, **kw):
    c = dict(kind="compact", pages=pages, used=used, batch=16, page_size=64, kv_heads=8, bits8=False,
             block=64, pinned=0)
    c.update(kw)
    return c


def listed():
    return [
        # the one new token of one request: latency is all there is
        dict(_norm(1, 2560), name="norm_token"),
        # a serving batch's tokens for products that take 8-bit rows (a scale for each)
        dict(_norm(333, 5120, group=5120, bf16=False), name="norm_rows8"),
        # a prompt chunk: bf16 for the projections here, and bytes in groups of 128 for 8-bit products
        dict(_norm(8192, 4096, group=128), name="norm_chunk"),
        # the backward pass of a short ragged batch, odd sizes
        dict(_grad(77, 1000), name="norm_grad_short"),
        # the backward pass of a training sequence
        dict(_grad(32768, 2560), name="norm_grad_train"),
        # one new token of each request of a serving batch, each with an adapter of its own or none
        dict(_adapt(32, 1, 4096, adapters=24), name="adapt_decode"),
        # a prompt chunk of one request behind its cache
        dict(_adapt(1, 8192, 16384, page_size=0), name="adapt_chunk"),
        # a few requests' chunks of odd lengths at once, larger rank, into the 8-bit cache (20 / 4 heads)
        dict(_adapt(5, 301, 2048, d=4096, rank=64, adapters=4, kv_heads=4, q_heads=20, bits8=True,
                    ragged=True), name="adapt_chunks8"),
        # one prompt answered twice: one page is copied
        dict(_fork(1, 2, 900, 1000), name="fork_pair"),
        # eight prompts with eight samples each, a 8-bit cache in pages of 128 tokens
        dict(_fork(8, 9, 4000, 30000, page_size=128, bits8=True), name="fork_samples"),
        # a small pool of which half is in use
        dict(_compact(200, 101, batch=3), name="compact_small"),
        # a pool after a day's requests came and went, some pages held from elsewhere
        dict(_compact(4096, 2600, batch=48, pinned=16), name="compact_pool"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same kinds and ranges."""
    what = rng.choice(["norm", "norm", "norm_grad", "adapt", "adapt_chunk", "fork", "compact"])
    heads = rng.choice([(32, 8), (32, 8), (20, 4), (16, 8), (8, 8)])
    if what in ("norm", "norm_grad"):
        d = rng.choice([512 * rng.randint(1, 16), 512 * rng.randint(1, 16), 8 * _log(rng, 8, 1024)])
        if what == "norm_grad":
            return _grad(_log(rng, 1, min(32768, 32768 * 2560 // d)), d, residual=rng.random() < 0.8)
        group = rng.choice([0, 32, 64, 128, 128, d])
        return _norm(_log(rng, 1, min(16384, 8192 * 4096 // d)), d, group=group,
                     bf16=group == 0 or rng.random() < 0.5, residual=rng.random() < 0.8)
    if what in ("adapt", "adapt_chunk"):
        page = rng.choice([0, 64, 128])
        kw = dict(d=512 * rng.randint(1, 12), rank=rng.choice([8, 16, 16, 32, 64, 128]),
                  adapters=_log(rng, 1, 64), q_heads=heads[0], kv_heads=heads[1], page_size=page,
                  bits8=rng.random() < 0.4, block=rng.choice([16, 32, 64]), ragged=rng.random() < 0.5)
        if what == "adapt":
            return _adapt(_log(rng, 1, 200), rng.choice([1, 1, rng.randint(2, 6)]), _log(rng, 64, 4096), **kw)
        batch = rng.randint(1, 6)
        t = _log(rng, 16, min(4096, 8192 * 2560 // (kw["d"] * batch)))
        return _adapt(batch, t, t + _log(rng, 1, 4096), **kw)
    page = rng.choice([16, 64, 64, 128, 256])
    kw = dict(page_size=page, kv_heads=heads[1], bits8=rng.random() < 0.5, block=min(page, rng.choice([16, 32, 64])))
    if what == "fork":
        prompts, samples = _log(rng, 1, 16), rng.randint(2, 9)
        hi = _log(rng, 100, min(32768, 200000 // prompts))
        return _fork(prompts, samples, rng.randint(hi // 2, hi), hi, n_q=rng.choice([1, 1, rng.randint(2, 300)]), **kw)
    pages = _log(rng, 50, 4096 * 64 // max(64, page))
    return _compact(pages, rng.randint(pages // 4, pages), batch=_log(rng, 1, 64),
                    pinned=rng.choice([0, 0, rng.randint(0, 8)]), **kw)


# ---- what the cases hold ----

def _normal(gen, shape, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEV).mul_(scale).to(BF16)


def _page_tensors(c, pages):
    """Shapes and types of what a page holds."""
    p, h, n = c["page_size"], c["kv_heads"], c["page_size"] // c["block"] if c["bits8"] else 0
    t = dict(k_idx=((pages, p, 4, IDX // 4), BF16))
    for w in "kv":
        t[w] = ((pages, p, h, D), E4M3 if c["bits8"] else BF16)
        if c["bits8"]:
            t[w + "_scale"] = ((pages, n, h), F32)
    if c["bits8"]:
        t["means"] = ((pages, n, IDX), BF16)
    return t


def _fill(gen, shape, dtype):
    if dtype == F32:
        return torch.exp2(torch.randint(-10, 3, shape, generator=gen, device=DEV).to(F32))
    x = torch.empty(shape, dtype=dtype, device=DEV)
    step = max(1, (1 << 26) // max(1, x[0].numel()))
    for i in range(0, shape[0], step):
        part = x[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV))
    return x


def _lens(c):
    """Tokens of each sequence or prompt: the longest first."""
    if c["kind"] == "fork":
        r = random.Random(c["prompts"] * 1000003 + c["len_lo"])
        return [c["len_hi"]] + [r.randint(c["len_lo"], c["len_hi"]) for _ in range(c["prompts"] - 1)]
    r = random.Random(c["batch"] * 1000003 + c["len_hi"])
    return [c["len_hi"]] + [r.randint(c["n_q"], c["len_hi"]) for _ in range(c["batch"] - 1)]


def _counts(c):
    """New tokens of each sequence of an adapt case."""
    r = random.Random(c["batch"] * 1009 + c["n_q"])
    return [c["n_q"] if i == 0 or not c["ragged"] else r.randint(0, c["n_q"]) for i in range(c["batch"])]


def _adapter_ids(c):
    r = random.Random(c["adapters"] * 7919 + c["batch"])
    return [0] + [r.randint(-1, c["adapters"] - 1) for _ in range(c["batch"] - 1)]


def _max_len(c):
    p = c["page_size"]
    most = c["len_hi"] + (c["n_q"] if c["kind"] == "fork" else 0)
    return -(-most // p) * p if p else most


def _fork_pages(c):
    """Pages that the prompts hold, and pages that the samples' new tokens take."""
    p, t = c["page_size"], c["n_q"]
    lens = _lens(c)
    return sum(-(-n // p) for n in lens), (c["samples"] - 1) * sum((n + t - 1) // p - n // p + 1 for n in lens)


def prepare(c, seed):
    """Inputs and output buffers of one case."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=c)
    kind = c["kind"]
    if kind in ("norm", "norm_grad"):
        n, d = c["rows"], c["d"]
        loud = torch.exp(0.7 * torch.randn(d, generator=gen, device=DEV))  # channels differ in size
        s["weight"] = (1 + 0.2 * torch.randn(d, generator=gen, device=DEV)).to(BF16)
        if kind == "norm":
            s["x"] = _normal(gen, (n, d))
            s["residual"] = (torch.randn((n, d), generator=gen, device=DEV) * loud * 3).to(BF16) if c["residual"] else None
            s["sum"] = torch.zeros((n, d), dtype=BF16, device=DEV) if c["residual"] else None
            s["y"] = torch.zeros((n, d), dtype=BF16, device=DEV) if c["bf16"] else None
            s["y8"] = s["y_scale"] = None
            if c["group"]:
                s["y8"] = torch.zeros((n, d), dtype=U8, device=DEV).view(E4M3)
                s["y_scale"] = torch.zeros((n, -(-d // c["group"])), device=DEV)
            s["rstd"] = torch.zeros(n, device=DEV)
            return s
        x = torch.randn((n, d), generator=gen, device=DEV) * loud
        s["s"] = x.to(BF16)
        s["rstd"] = (s["s"].to(F64).square().mean(1) + EPS).rsqrt().to(F32) if n * d < 1 << 24 else \
            (s["s"].to(F32).square().mean(1) + EPS).rsqrt()
        s["dy"] = _normal(gen, (n, d), 1e-3)
        s["dsum"] = _normal(gen, (n, d), 1e-3) if c["residual"] else None
        s["dx"] = torch.zeros((n, d), dtype=BF16, device=DEV)
        s["dweight"] = torch.zeros(d, device=DEV)
        return s
    p = c["page_size"]
    if kind == "adapt":
        bt, t, d, h, r, m = c["batch"], c["n_q"], c["d"], c["kv_heads"], c["rank"], c["adapters"]
        feats = 2 * IDX + 2 * h * D
        s["h"] = _normal(gen, (bt, t, d))
        s["w"] = _normal(gen, (feats, d), 1 / math.sqrt(d))
        s["a"] = _normal(gen, (m, r, d), 1 / math.sqrt(d))
        s["b"] = _normal(gen, (m, feats, r), 0.1)
        s["alpha"] = torch.rand(m, generator=gen, device=DEV) * 2
        s["adapter"] = torch.tensor(_adapter_ids(c), dtype=I32, device=DEV)
        lens, new = _lens(c), _counts(c)
        start = [n - t for n in lens]
        s["start"] = torch.tensor(start, dtype=I32, device=DEV)
        s["count"] = torch.tensor(new, dtype=I32, device=DEV)
        # rows behind a sequence's last new token have no place in the cache
        s["pos"] = torch.tensor([[a + i if i < k else -1 for i in range(t)] for a, k in zip(start, new)],
                                dtype=I32, device=DEV)
        s["page_table"] = None
        if p:
            need = [-(-n // p) for n in lens]
            perm = torch.randperm(sum(need), generator=gen, device=DEV).to(I32)
            s["page_table"] = torch.full((bt, _max_len(c) // p), -1, dtype=I32, device=DEV)
            at = 0
            for b, n in enumerate(need):
                s["page_table"][b, :n] = perm[at:at + n]
                at += n
            rows, blocks = (sum(need), p), (sum(need), p // c["block"])
        else:
            rows, blocks = (bt, _max_len(c)), (bt, -(-_max_len(c) // c["block"]))
        s["q_idx"] = torch.zeros((bt, t, 4, IDX // 4), dtype=BF16, device=DEV)
        s["k_idx"] = _fill(gen, rows + (4, IDX // 4), BF16)
        for w in "kv":
            s[w] = _fill(gen, rows + (h, D), E4M3 if c["bits8"] else BF16)
            if c["bits8"]:
                s[w + "_scale"] = torch.exp2(torch.randint(-9, -6, blocks + (h,), generator=gen, device=DEV).to(F32))
        return s
    if kind == "fork":
        held, more = _fork_pages(c)
        pages, n = held + more + held // 8 + 3, c["samples"]
        bt = c["prompts"] * n
        lens = [x for m in _lens(c) for x in [m] + [0] * (n - 1)]
        s["parent"] = torch.arange(bt, device=DEV, dtype=I32) // n * n
        s["count"] = torch.tensor([0 if b % n == 0 else c["n_q"] for b in range(bt)], dtype=I32, device=DEV)
    else:
        pages, bt = c["pages"], c["batch"]
        # sequences of unequal lengths, every fourth one holding the first page of the one before it
        r = random.Random(pages * 31 + bt)
        cuts = sorted(r.randint(0, c["used"]) for _ in range(bt - 1))
        lens = [p * (b - a) for a, b in zip([0] + cuts, cuts + [c["used"]])]
    s["tensors"] = {k: _fill(gen, *v) for k, v in _page_tensors(c, pages).items()}
    need = [-(-n // p) for n in lens]
    cols = _max_len(c) // p if kind == "fork" else max(need) + 1
    perm = torch.randperm(pages, generator=gen, device=DEV).to(I32)
    s["page_table"] = torch.full((bt, cols), -1, dtype=I32, device=DEV)
    s["refs"] = torch.zeros(pages, dtype=I32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        s["page_table"][b, :n] = perm[at:at + n]
        at += n
        if kind == "compact" and b % 4 == 3 and need[b - 1]:
            s["page_table"][b, n] = s["page_table"][b - 1, 0]
    held = s["page_table"].flatten().long()
    s["refs"].index_add_(0, held.clamp(min=0), (held >= 0).to(I32))
    if kind == "compact":
        s["refs"][perm[:min(c["pinned"], c["used"])].long()] += 1
        s["table_then"], s["refs_then"] = s["page_table"].clone(), s["refs"].clone()
        s["bound"] = torch.zeros(1, dtype=I32, device=DEV)
        s["max_len"] = cols * p
    else:
        s["seq_lens"] = torch.tensor(lens, dtype=I32, device=DEV)
        s["missing"] = torch.zeros(1, dtype=I32, device=DEV)
        s["max_len"] = _max_len(c)
    return s


# ---- plain forms ----

def _scale_of(a):
    """The least power of two that holds magnitude a within 448 times it."""
    m, e = torch.frexp(a)                                       # 448 = 0.875 * 2^9
    e = torch.where(a > 0, e - 9 + (m > 0.875).to(e.dtype), E_MIN).clamp(min=E_MIN)
    return torch.ldexp(torch.ones_like(a), e)


def _plain_norm(s):
    c = s["case"]
    x = s["x"]
    if c["residual"]:
        x = (x.to(F32) + s["residual"].to(F32)).to(BF16)
    # the sum decides, through its one rounding, next to a border of a scale: 64 bits
    rstd = (1 / torch.sqrt(x.to(F64).square().mean(1) + EPS)).to(F32)
    y = x.to(F32) * rstd[:, None] * s["weight"].to(F32)
    r = dict(rstd=rstd)
    if c["residual"]:
        r["sum"] = x
    if c["bf16"]:
        r["y"] = y.to(BF16)
    if c["group"]:
        n = c["group"]
        groups = -(-c["d"] // n)
        z = torch.nn.functional.pad(y, (0, groups * n - c["d"])).view(-1, groups, n)
        scale = _scale_of(z.abs().amax(2))
        r["y8"] = (z / scale[..., None]).to(E4M3).view(U8).view(-1, groups * n)[:, :c["d"]].contiguous().view(E4M3)
        r["y_scale"] = scale
    return r


def _plain_grad(s):
    dy, x = s["dy"].to(F32), s["s"].to(F32) * s["rstd"][:, None]
    g = dy * s["weight"].to(F32)
    dx = (g - x * (g * x).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["dsum"] is not None:
        dx += s["dsum"].to(F32)
    return dict(dx=dx.to(BF16), dweight=(dy * x).sum(0, dtype=F64).to(F32))


def _token_rows(s, b, j):
    """Row of token j of sequence b in a cache seen as [tokens, ...] (j: int64)."""
    p = s["case"]["page_size"]
    if not p:
        return b * _max_len(s["case"]) + j
    return s["page_table"][b, j // p].long() * p + j % p


def _block_rows(s, b, blk):
    p, n = s["case"]["page_size"], s["case"]["block"]
    if not p:
        return b * (-(-_max_len(s["case"]) // n)) + blk
    return s["page_table"][b, blk * n // p].long() * (p // n) + blk * n % p // n


def _append8(s, what, rows):
    """New rows [batch, n_q, heads, D] (bf16 values) into the 8-bit cache."""
    c = s["case"]
    n, h, last = c["block"], c["kv_heads"], _max_len(c) - 1
    start, count = s["start"].long(), s["count"].long()
    b = torch.arange(c["batch"], device=DEV)[:, None]
    most = (c["n_q"] + n - 2) // n + 1
    # blocks that the new tokens reach, a sequence's last one in the place of those past it
    blk = torch.minimum(start[:, None] // n + torch.arange(most, device=DEV), ((start + count - 1).clamp(min=0) // n)[:, None])
    pos = blk[..., None] * n + torch.arange(n, device=DEV)      # [batch, blocks, n]
    first, end = start[:, None, None], (start + count)[:, None, None]
    new, kept = (pos >= first) & (pos < end), pos < first
    x = rows[b[..., None], (pos - first).clamp(0, c["n_q"] - 1)].to(F32)
    fresh = _scale_of(torch.where(new[..., None, None], x, 0).abs().amax((2, 4)))
    scales, at = s[what + "_scale"].view(-1, h), _block_rows(s, b, blk)
    old = scales[at]
    sc = torch.where(kept.any(-1)[..., None], torch.maximum(old, fresh), fresh)
    sc = torch.where((count > 0)[:, None, None], sc, old)
    byte = s[what].view(U8).view(-1, h, D)
    # the last block of a cache whose length is no multiple of n ends early
    at_row = _token_rows(s, b[..., None], pos.clamp(max=last))
    was = byte[at_row]
    moved = (was.view(E4M3).to(F32) * (old / sc)[:, :, None, :, None]).to(E4M3).view(U8)
    put = (x / sc[:, :, None, :, None]).to(E4M3).view(U8)
    now = torch.where(new[..., None, None], put, torch.where(kept[..., None, None], moved, was))
    if (last + 1) % n:  # rows past the end repeat the last token's
        i = last % n
        now = torch.where((pos <= last)[..., None, None], now, now[:, :, i:i + 1])
    byte[at_row] = now
    scales[at] = sc


def _plain_adapt(s):
    c = s["case"]
    bt, t, h = c["batch"], c["n_q"], c["kv_heads"]
    x = s["h"].to(F32)
    out = (x.view(bt * t, -1) @ s["w"].to(F32).t()).view(bt, t, -1)
    ad = s["adapter"].long()
    held = ad.clamp(min=0)
    u = torch.bmm(x, s["a"][held].to(F32).transpose(1, 2).contiguous()) * s["alpha"][held][:, None, None]
    more = torch.bmm(u, s["b"][held].to(F32).transpose(1, 2).contiguous())
    out = torch.where((ad >= 0)[:, None, None], out + more, out).to(BF16)
    q, ki, k, v = out.split([IDX, IDX, h * D, h * D], 2)
    s["q_idx"].copy_(q.reshape(s["q_idx"].shape))
    live = s["pos"] >= 0
    b = torch.arange(bt, device=DEV)[:, None].expand(bt, t)
    rows = _token_rows(s, b[live], s["pos"][live].long())
    s["k_idx"].view(-1, IDX)[rows] = ki[live]
    if c["bits8"]:
        _append8(s, "k", k.reshape(bt, t, h, D))
        _append8(s, "v", v.reshape(bt, t, h, D))
    else:
        s["k"].view(-1, h * D)[rows] = k[live]
        s["v"].view(-1, h * D)[rows] = v[live]
    return _adapted(s)


def _adapted(s):
    return {k: s[k] for k in ("q_idx", "k_idx", "k", "v", "k_scale", "v_scale") if k in s}


def _plain_fork(s):
    c, table, refs = s["case"], s["page_table"], s["refs"]
    # fork
    old = table.clone()
    up = s["parent"].long()
    table.copy_(torch.where(up[:, None] >= 0, old[up.clamp(min=0)], -1))
    s["seq_lens"].copy_(torch.where(up >= 0, s["seq_lens"][up.clamp(min=0)], 0))
    refs.index_add_(0, table.flatten().long().clamp(min=0), (table >= 0).flatten().to(I32))
    refs.index_add_(0, old.flatten().long().clamp(min=0), -(old >= 0).flatten().to(I32))
    # reserve
    p, bt, pages = c["page_size"], table.shape[0], refs.numel()
    start, end = s["seq_lens"].long(), (s["seq_lens"] + s["count"]).long()
    slot = torch.arange((c["n_q"] + p - 2) // p + 1, device=DEV)
    at = start[:, None] // p + slot
    touched = (at * p < end[:, None]) & (s["count"] > 0)[:, None]
    at = at.clamp(max=table.shape[1] - 1)
    b = torch.arange(bt, device=DEV)[:, None].expand(at.shape)
    e = table[b, at].long()
    writer = touched & (e >= 0)
    order = torch.arange(at.numel(), device=DEV).view(at.shape)
    held = torch.where(writer, e, pages)                        # a place of its own for the others
    writers = torch.zeros(pages + 1, dtype=I32, device=DEV)
    writers.index_add_(0, held.flatten(), torch.ones_like(held.flatten(), dtype=I32))
    last = torch.full((pages + 1,), -1, device=DEV).scatter_reduce_(0, held.flatten(), order.flatten(), "amax")
    holders = torch.nn.functional.pad(refs, (0, 1))
    # where every holder of a page writes, the last of them keeps it
    keeps = writer & (writers[held] == holders[held]) & (order == last[held])
    copies = writer & ~keeps
    need = (touched & (e < 0)) | copies
    free = torch.sort((refs != 0).to(U8), stable=True).indices
    s["missing"].copy_((need.sum() - (refs == 0).sum()).clamp(min=0))
    enough = s["missing"] == 0
    need, copies = need & enough, copies & enough
    new = free[(need.flatten().cumsum(0) - 1).clamp(min=0, max=pages - 1)].view(at.shape)
    refs.index_add_(0, e.clamp(min=0).flatten(), -copies.flatten().to(I32))
    refs[new[need]] = 1
    table[b[need], at[need]] = new[need].to(I32)
    [x.view(U8).view(pages, -1).index_copy_(0, new[copies], x.view(U8).view(pages, -1)[e[copies]])
     for x in s["tensors"].values()]
    return _forked(s)


def _forked(s):
    return dict(page_table=s["page_table"], seq_lens=s["seq_lens"], refs=s["refs"], missing=s["missing"], **s["tensors"])


def _plain_compact(s):
    table, refs = s["page_table"], s["refs"]
    pages = refs.numel()
    held = table.flatten().long()
    count = torch.zeros(pages, dtype=I32, device=DEV).index_add_(0, held.clamp(min=0), (held >= 0).to(I32))
    page = torch.arange(pages, device=DEV)
    used = refs > 0
    total = used.sum()
    # a page that something beside the table refers to stays where it is
    move = used & (refs == count) & (page >= total)
    hole = ~used & (page < total)
    src, dst = page[move], page[hole][:int(move.sum())]
    to = page.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table))
    refs[dst] = refs[src]
    refs[src] = 0
    s["bound"].copy_(torch.where(refs > 0, page + 1, 0).amax())
    [x.view(U8).view(pages, -1).index_copy_(0, dst, x.view(U8).view(pages, -1)[src]) for x in s["tensors"].values()]
    return _compacted(s)


def _compacted(s):
    return dict(page_table=s["page_table"], refs=s["refs"], bound=s["bound"], **s["tensors"])


def _before(s):
    """A compacted pool has nothing left to move: a pass starts with the tables as they were (the
    pages that move hold what they held, and the ones that they move to are written over)."""
    if s["case"]["kind"] == "compact":
        s["page_table"].copy_(s["table_then"])
        s["refs"].copy_(s["refs_then"])


def _plain(s):
    return dict(norm=_plain_norm, norm_grad=_plain_grad, adapt=_plain_adapt, fork=_plain_fork,
                compact=_plain_compact)[s["case"]["kind"]](s)


# ---- the library's calls ----

def _handles(s):
    """The shape and workspace that a program keeps beside its buffers."""
    from paper_2606_06467_amd import binding as B
    if "shape" not in s:
        c = s["case"]
        kind, ws = c["kind"], None
        if kind in ("norm", "norm_grad"):
            s["shape"] = B.make_shape(c["rows"], 1, 1, 1)
            if kind == "norm_grad":
                ws = B.CLSA_OP_NORM_GRAD, c["d"]
        elif kind == "adapt":
            m, p = _max_len(c), c["page_size"]
            s["shape"] = B.make_shape(c["batch"], c["n_q"], m, 1, q_heads=c["q_heads"], kv_heads=c["kv_heads"],
                                      page_size=p, max_pages=m // p if p else 0)
            ws = B.CLSA_OP_ADAPTED8 if c["bits8"] else B.CLSA_OP_ADAPTED, c["rank"]
        else:
            bt, cols = s["page_table"].shape
            s["shape"] = B.make_shape(bt, c.get("n_q", 1), s["max_len"], 1, page_size=c["page_size"], max_pages=cols)
            s["list"] = list(s["tensors"].values())
            ws = (B.CLSA_OP_PAGES_RESERVE, 0) if kind == "fork" else (B.CLSA_OP_PAGES_COMPACT, c["pages"])
        s["ws"] = B.workspace(s["shape"], *ws, DEV) if ws else None
    return B, s["shape"]


def _library(s):
    c = s["case"]
    kind = c["kind"]
    B, sh = _handles(s)
    if kind == "norm":
        B.clsa_residual_norm(sh, c["d"], EPS, s["x"], s["residual"], s["weight"], s["sum"], s["y"], s["y8"],
                             s["y_scale"], s["rstd"], group=c["group"])
        return {k: s[k] for k in ("rstd", "sum", "y", "y8", "y_scale") if s[k] is not None}
    if kind == "norm_grad":
        B.clsa_residual_norm_grad(sh, c["d"], s["s"], s["rstd"], s["weight"], s["dy"], s["dsum"], s["dx"],
                                  s["dweight"], s["ws"])
        return dict(dx=s["dx"], dweight=s["dweight"])
    if kind == "adapt":
        lora = s["a"], s["b"], s["alpha"], s["adapter"]
        if c["bits8"]:
            B.clsa_project_append8_adapted(sh, c["block"], c["d"], s["h"], s["w"], *lora, s["start"], s["count"],
                                           s["page_table"], s["q_idx"], s["k_idx"], s["k"], s["v"], s["k_scale"],
                                           s["v_scale"], s["ws"])
        else:
            B.clsa_project_append_adapted(sh, c["d"], s["h"], s["w"], *lora, s["pos"], s["page_table"], s["q_idx"],
                                          s["k_idx"], s["k"], s["v"], s["ws"])
        return _adapted(s)
    if kind == "fork":
        B.clsa_pages_fork(sh, s["parent"], s["page_table"], s["seq_lens"], s["refs"])
        B.clsa_pages_reserve(sh, s["list"], s["seq_lens"], s["count"], s["page_table"], s["refs"], s["missing"], s["ws"])
        return _forked(s)
    B.clsa_pages_compact(sh, s["list"], s["page_table"], s["refs"], s["bound"], s["ws"])
    return _compacted(s)


def run(s):
    _before(s)
    return _library(s) if own else _plain(s)


def _page_bytes(c):
    return sum(math.prod(shape) * dtype.itemsize for shape, dtype in _page_tensors(c, 1).values())


def work(c):
    kind = c["kind"]
    if kind == "norm":
        n, d = c["rows"], c["d"]
        each = 2 + (4 if c["residual"] else 0) + (2 if c["bf16"] else 0) + (1 if c["group"] else 0)
        return dict(bytes=n * d * each + 2 * d + 4 * n + (4 * n * -(-d // c["group"]) if c["group"] else 0),
                    flops=6 * n * d)
    if kind == "norm_grad":
        n, d = c["rows"], c["d"]
        return dict(bytes=n * d * (8 if c["residual"] else 6) + 6 * d + 4 * n, flops=10 * n * d)
    if kind == "adapt":
        bt, t, d, r = c["batch"], c["n_q"], c["d"], c["rank"]
        feats, ids = 2 * IDX + 2 * c["kv_heads"] * D, _adapter_ids(c)
        one, new = len({i for i in ids if i >= 0}), sum(_counts(c))
        adapted = sum(t for i in ids if i >= 0)
        kv = 2 * c["kv_heads"] * D * (1 if c["bits8"] else 2)
        return dict(bytes=2 * d * (feats + bt * t) + 2 * one * r * (d + feats) + 2 * IDX * (bt * t + new) + new * kv,
                    flops=2 * bt * t * d * feats + 2 * adapted * r * (d + feats))
    if kind == "fork":
        cols = _max_len(c) // c["page_size"]
        rows = c["prompts"] * c["samples"]
        held, more = _fork_pages(c)
        p, t = c["page_size"], c["n_q"]
        shared = [n for n in _lens(c) if n % p]                 # prompts whose last page is copied
        return dict(bytes=rows * cols * 8 + 8 * (held + more) + len(shared) * c["samples"] * _page_bytes(c),
                    flops=rows * cols)
    move = c["used"] * (c["pages"] - c["used"]) / c["pages"]    # as many as there are holes, on average
    return dict(bytes=2 * move * _page_bytes(c) + 8 * c["pages"] + 16 * c["used"], flops=c["pages"])


# ---- the definitions in 64 bits ----

def _exact_norm(s):
    c, d = s["case"], s["case"]["d"]
    x = s["x"].double()
    if c["residual"]:
        x = (x + s["residual"].double()).to(F32).to(BF16).double()
    rstd = torch.rsqrt((x * x).sum(-1) / d + EPS)
    y = x * rstd.unsqueeze(-1) * s["weight"].double()
    r = dict(rstd=rstd)
    if c["residual"]:
        r["sum"] = s["x"].double() + s["residual"].double()
    if c["bf16"]:
        r["y"] = y
    if c["group"]:
        parts = y.split(c["group"], 1)
        sc = [torch.exp2(torch.ceil(torch.log2(p.abs().amax(1, keepdim=True) / 448)).clamp(min=E_MIN)) for p in parts]
        r["y_scale"] = torch.cat(sc, 1)
        r["y8"] = torch.cat([p / f for p, f in zip(parts, sc)], 1)
    return r


def _exact_grad(s):
    dx, dw = [], 0
    w = s["weight"].double()
    for i in range(0, s["s"].shape[0], 4096):
        rows = slice(i, i + 4096)
        x, dy, r = s["s"][rows].double(), s["dy"][rows].double(), s["rstd"][rows, None].double()
        dot = (dy * w * x).sum(1, keepdim=True) / x.shape[1]
        one = r * dy * w - x * r ** 3 * dot
        dx.append(one if s["dsum"] is None else one + s["dsum"][rows].double())
        dw = dw + (dy * (x * r)).sum(0)
    return dict(dx=torch.cat(dx), dweight=dw)


def _exact_adapt(s):
    c = s["case"]
    bt, t, h, n, p = c["batch"], c["n_q"], c["kv_heads"], c["block"], c["page_size"]
    r = {k: v.to(F32).double() if v.dtype == E4M3 else v.double() for k, v in _adapted(s).items()}
    w = s["w"].double()
    for i, ad in enumerate(_adapter_ids(c)):
        full = w if ad < 0 else w + s["alpha"][ad].double() * (s["b"][ad].double() @ s["a"][ad].double())
        out = s["h"][i].double() @ full.t()
        r["q_idx"][i] = out[:, :IDX].view(t, 4, IDX // 4)
        first, m = int(s["start"][i]), _counts(c)[i]
        if not m:
            continue
        j = torch.arange(first, first + m, device=DEV)
        at = (s["page_table"][i, j // p].long(), j % p) if p else (torch.full_like(j, i), j)
        r["k_idx"][at] = out[:m, IDX:2 * IDX].view(m, 4, IDX // 4)
        for k, what in enumerate("kv"):
            x = out[:m, 2 * IDX + k * h * D:2 * IDX + (k + 1) * h * D].view(m, h, D)
            if not c["bits8"]:
                r[what][at] = x
                continue
            x = x.to(F32).to(BF16).double()                      # the cache takes rows rounded to bf16
            for blk in range(first // n, -(-(first + m) // n)):
                lo, hi = max(first, blk * n), min(first + m, blk * n + n)
                top = x[lo - first:hi - first]
                need = torch.exp2(torch.ceil(torch.log2(top.abs().amax((0, 2)) / 448)))
                row, off = (int(s["page_table"][i, blk * n // p]), blk * n % p) if p else (i, blk * n)
                have = r[what + "_scale"][row, off // n].clone()
                sc = torch.maximum(have, need) if lo > blk * n else need
                r[what][row, off:off + lo - blk * n] *= (have / sc)[:, None]
                r[what][row, off + lo - blk * n:off + hi - blk * n] = top / sc[:, None]
                r[what + "_scale"][row, off // n] = sc
    return r


def exact(c, seed):
    """What run() returns for these inputs, from the definitions in 64 bits; pages move whole."""
    if c["kind"] in ("fork", "compact"):
        return None
    s = prepare(c, seed)
    return dict(norm=_exact_norm, norm_grad=_exact_grad, adapt=_exact_adapt)[c["kind"]](s)
