"""Plain references of the calls on pages: one entry after another, in Python's integers."""
from __future__ import annotations

import numpy as np


def holders(table, pages):
    """How many entries of the table name each page."""
    e = table[(table >= 0) & (table < pages)]
    return np.bincount(e, minlength=pages).astype(np.int32)


def fork(parent, table, lens, refs):
    """(table, lens, refs, whether a number was out of range) after clsa_pages_fork."""
    t, l, r, bad = table.copy(), lens.copy(), refs.copy(), False
    pages = len(refs)
    for b, up in enumerate(parent):
        if up < -1 or up >= len(parent):
            bad = True
        elif up != b:
            l[b] = 0 if up < 0 else lens[up]
            for c in range(table.shape[1]):
                old, new = int(table[b, c]), -1 if up < 0 else int(table[up, c])
                bad |= not (-1 <= old < pages and -1 <= new < pages)
                new = new if 0 <= new < pages else -1
                if new == old:
                    continue
                t[b, c] = new
                if new >= 0:
                    r[new] += 1
                if 0 <= old < pages:
                    r[old] -= 1
    return t, l, r, bad


def reserve(start, count, table, refs, n_q, page, max_len):
    """(table, refs, copies [(from, to)], missing) after clsa_pages_reserve.

    Entries are taken in order; a page that has one holder left is written in place: its
    other holders have got copies, or never had it."""
    t, r = table.copy(), refs.copy()
    pages = len(refs)
    entries = []
    for b in range(len(start)):
        n = min(max(int(count[b]), 0), n_q)
        if 0 <= start[b] <= max_len:
            end = int(start[b]) + min(n, max_len - int(start[b]))
            if end > start[b]:
                entries += [(b, p) for p in range(int(start[b]) // page, (end - 1) // page + 1)]
    free = iter(np.flatnonzero(refs == 0).tolist())
    need, copies = 0, []
    for b, p in entries:
        e = int(t[b, p])
        held = 0 <= e < pages
        if held and r[e] == 1:
            continue
        need += 1
        to = next(free, None)
        if to is None:
            continue
        if held:
            r[e] -= 1
            copies.append((e, to))
        t[b, p] = to
        r[to] = 1
    lack = max(0, need - int((refs == 0).sum()))
    if lack:
        # what a full pool changes: nothing.  The number that lacks counts every need, also
        # those past the point where the loop above ran out of pages
        return table.copy(), refs.copy(), [], _needs(entries, table, refs) - int((refs == 0).sum())
    return t, r, copies, 0


def _needs(entries, table, refs):
    r, n = refs.copy(), 0
    for b, p in entries:
        e = int(table[b, p])
        if 0 <= e < len(refs):
            if r[e] == 1:
                continue
            r[e] -= 1
        n += 1
    return n


def compact(table, refs):
    """(table, refs, moves [(from, to)], bound) after clsa_pages_compact."""
    t, r = table.copy(), refs.copy()
    pages = len(refs)
    held = holders(table, pages)
    used = int((refs > 0).sum())
    holes = iter([p for p in range(used) if refs[p] <= 0])
    moves = []
    for p in range(used, pages):
        if refs[p] > 0 and refs[p] == held[p]:
            to = next(holes)
            moves.append((p, to))
            r[to], r[p] = refs[p], 0
            t[table == p] = to
    live = np.flatnonzero(r > 0)
    return t, r, moves, int(live[-1]) + 1 if len(live) else 0


def state(rng, batch, cols, pages, fill=0.6, shared=0.5, pinned=0, bad=0.0):
    """A table, lengths in pages, and refs: sequences with pages of their own, some sharing a prefix."""
    free = rng.permutation(pages).tolist()
    table = np.full((batch, cols), -1, np.int32)
    for b in range(batch):
        n, at = int(rng.integers(0, cols + 1) * fill), 0
        if b and rng.random() < shared:
            src = int(rng.integers(0, b))
            at = min(n, int(rng.integers(0, cols + 1)))
            at = min(at, int((table[src] >= 0).sum()))
            table[b, :at] = table[src, :at]
        for c in range(at, n):
            if not free:
                break
            table[b, c] = free.pop()
    refs = holders(table, pages)
    for p in rng.permutation(pages)[:pinned]:
        refs[p] += 1
    if bad:
        wrong = rng.random(table.shape) < bad
        refs -= holders(np.where(wrong, table, -1), pages)
        table[wrong] = rng.choice([-7, pages, pages + 5, 2 ** 31 - 1, -2 ** 31], int(wrong.sum()))
    return table, refs
