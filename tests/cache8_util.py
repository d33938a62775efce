"""Plain references of the 8-bit cache and of block routing for the tests, in 64 bits.

The e4m3 table is made from the format's definition; rounding picks the nearest entry,
ties to the even mantissa."""
from __future__ import annotations

import numpy as np

from paper_2606_06467_amd import inputs

D = 128
TOP = 240.0 * 2.0 ** 120


def _table():
    v = np.zeros(127)
    for b in range(127):  # 0x7f is NaN
        e, m = b >> 3, b & 7
        v[b] = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
    return v


E4M3 = _table()
VALUES = np.concatenate([E4M3, [np.nan], -E4M3, [np.nan]])  # by byte


def encode(x: np.ndarray) -> np.ndarray:
    """e4m3 bytes of values within +-448 (NaN and infinities: NaN), nearest, ties to even."""
    a = np.abs(np.asarray(x, np.float64))
    bad = ~np.isfinite(a)
    a = np.where(bad, 0.0, a)
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)
    lo = hi - 1
    up, down = E4M3[hi] - a, a - E4M3[lo]
    b = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    b = b | np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(bad, 0x7f, b).astype(np.uint8)


def same_bytes(a, b):
    """Equal, where every NaN is alike."""
    nan_a, nan_b = (a & 0x7f) == 0x7f, (b & 0x7f) == 0x7f
    return np.array_equal(nan_a, nan_b) and np.array_equal(a[~nan_a], b[~nan_a])


class Cache:
    """K (or V) bytes and scales, addressed by (sequence, token), contiguous or paged."""

    def __init__(self, batch, max_len, heads, block, page_size=0, page_table=None, fill=0x55):
        self.block, self.page, self.pt, self.max_len = block, page_size, page_table, max_len
        if page_size:
            pages = int(page_table.max()) + 1
            self.bytes = np.full((pages, page_size, heads, D), fill, np.uint8)
            self.scale = np.full((pages, page_size // block, heads), 1.0, np.float32)
        else:
            self.bytes = np.full((batch, max_len, heads, D), fill, np.uint8)
            self.scale = np.full((batch, -(-max_len // block), heads), 1.0, np.float32)

    def at(self, b, j):
        return (b, j) if not self.page else (int(self.pt[b, j // self.page]), j % self.page)

    def block_at(self, b, c):
        if not self.page:
            return (b, c)
        j = c * self.block
        return int(self.pt[b, j // self.page]), j % self.page // self.block

    def append(self, b, start, x):
        """Rows x [n, heads, D] (float64) at positions start..."""
        n, s = len(x), self.block
        for c in range(start // s, -(-(start + n) // s)):
            lo, hi = max(start, c * s), min(start + n, c * s + s)
            new = np.clip(x[lo - start:hi - start], -TOP, TOP)
            new[~np.isfinite(x[lo - start:hi - start])] = np.nan
            a = np.nan_to_num(np.abs(new), nan=0.0).max((0, 2))
            e = np.full(a.shape, -100.0)
            for h in range(len(a)):
                while a[h] > 448 * 2.0 ** e[h]:
                    e[h] += 1
            fresh, at = 2.0 ** e, self.block_at(b, c)
            keeps = lo > c * s
            old = self.scale[at].astype(np.float64)
            now = np.maximum(old, fresh) if keeps else fresh
            if keeps:
                for j in range(c * s, lo):
                    p = self.at(b, j)
                    for h in np.nonzero(now > old)[0]:
                        self.bytes[p][h] = encode(VALUES[self.bytes[p][h]] * (old[h] / now[h]))
            for j in range(lo, hi):
                self.bytes[self.at(b, j)] = encode(new[j - lo] / now[:, None])
            self.scale[at] = now

    def values(self):
        """Every cached value, in the layout of the bytes."""
        s = np.repeat(self.scale.astype(np.float64), self.block, axis=1)[:, :self.bytes.shape[1]]
        return VALUES[self.bytes] * s[..., None]

    def rows(self, b, n):
        """Values of the first n tokens of sequence b."""
        v = self.values()
        return np.stack([v[self.at(b, j)] for j in range(n)]) if n else np.zeros((0,) + v.shape[2:])


def filled(seed, lens, heads, block, max_len, page_size=0, page_table=None):
    """A cache filled with random rows, blocks of different sizes; the rest of it holds NaN."""
    g = np.random.default_rng(seed)
    c = Cache(len(lens), max_len, heads, block, page_size, page_table, fill=0x7f)
    for b, n in enumerate(lens):
        x = g.standard_normal((n, heads, D)) * 2.0 ** g.integers(-3, 4, size=(-(-n // block), heads)) \
            .repeat(block, 0)[:n, :, None]
        if n:
            for k in range(0, n, block):  # vectorised: whole blocks
                y = x[k:k + block]
                e = np.ceil(np.log2(np.abs(y).max((0, 2)) / 448))
                c.scale[c.block_at(b, k // block)] = 2.0 ** e
                p = c.at(b, k)
                c.bytes[p[0], p[1]:p[1] + len(y)] = encode(y / 2.0 ** e[:, None])
    return c


def page_table(seed, lens, page, max_len):
    need = [-(-n // page) for n in lens]
    perm = np.random.default_rng(seed).permutation(max(1, sum(need))).astype(np.int32)
    pt = np.full((len(lens), max_len // page), -1, np.int32)
    at = 0
    for b, m in enumerate(need):
        pt[b, :m] = perm[at:at + m]
        at += m
    return pt


def attention(q, kc, vc, sets, scale):
    """Softmax attention of q [B, T, Hq, D] (float64) over the tokens sets[b][t]: out, lse, and
    tolerances of both.

    A weight reaches the second product as bf16 (half a step is 2^-8 of it) and so does the
    result; a logit of 128 fp32 products is off by at most 128 * 2^-23 of their magnitudes, and
    the exponential, logarithm and the scale's product by a few fp32 steps (2^-20)."""
    B, T, Hq, _ = q.shape
    H = kc.bytes.shape[2]
    G = Hq // H
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    t_out, t_lse = np.zeros(q.shape), np.zeros(q.shape[:3])
    kv, vv = kc.values(), vc.values()
    for b in range(B):
        for t in range(T):
            s = sets[b][t]
            if len(s) == 0:
                continue
            at = [kc.at(b, int(j)) for j in s]
            i0, i1 = np.array([p[0] for p in at]), np.array([p[1] for p in at])
            k, v = kv[i0, i1], vv[i0, i1]  # [n, H, D]
            for h in range(Hq):
                kh, vh = k[:, h // G], v[:, h // G]
                z = kh @ q[b, t, h] * scale
                d = 2.0 ** -16 * (np.abs(kh) @ np.abs(q[b, t, h])) * abs(scale)
                m = z.max()
                w = np.exp(z - m)
                total = w.sum()
                w = w / total
                out[b, t, h] = w @ vh
                lse[b, t, h] = m + np.log(total)
                err = 2 * d + 2.0 ** -20 * (1 + np.abs(z - m))
                t_out[b, t, h] = ((w * (2.0 ** -8 + 2 * err)) @ np.abs(vh) + 2.0 ** -8 * np.abs(out[b, t, h]) +
                                  2 * (w @ err) * np.abs(out[b, t, h])) * 1.01 + 1e-30
                t_lse[b, t, h] = d.max() + 2.0 ** -20 * (1 + abs(lse[b, t, h]))
    return out, lse, t_out, t_lse


def check_attention(got, got_lse, want):
    """got: bf16 bits; got_lse: fp32."""
    out, lse, t_out, t_lse = want
    o = inputs.f32_from_bf16_bits(got).astype(np.float64)
    nan = np.isnan(out)
    assert np.array_equal(np.isnan(o), nan), "NaN in other places"
    off = np.abs(o - out)[~nan] / np.where(t_out[~nan] > 0, t_out[~nan], 1.0)
    assert off.size == 0 or off.max() <= 1.0, f"output off by {off.max():.3f} of its tolerance"
    if got_lse is not None:
        assert np.array_equal(np.isnan(got_lse), np.isnan(lse))
        fin = np.isfinite(lse)
        assert np.array_equal(got_lse[~fin & ~np.isnan(lse)], lse[~fin & ~np.isnan(lse)])
        off = np.abs(got_lse - lse)[fin] / t_lse[fin]
        assert off.size == 0 or off.max() <= 1.0, f"lse off by {off.max():.3f} of its tolerance"


def route(q, means, n, block, top_k):
    """Token list of one row: q [256], means [blocks, 256] in float64, n valid keys."""
    out = np.full(top_k, -1, np.int32)
    if n == 0:
        return out, 0
    own, want = (n - 1) // block, top_k // block - 1
    s = np.array([float(np.dot(q, means[c])) for c in range(own)])
    best = np.sort(np.argsort(-s, kind="stable")[:want]) if own else np.zeros(0, int)
    tok = np.concatenate([np.arange(c * block, (c + 1) * block) for c in best] +
                         [np.arange(own * block, n)])
    out[:len(tok)] = tok
    return out, len(tok)


def bf16(a):
    """float64 values of an array rounded to bf16, and its bits."""
    bits = inputs.bf16_bits_from_f32(np.asarray(a, np.float32))
    return inputs.f32_from_bf16_bits(bits).astype(np.float64), bits
