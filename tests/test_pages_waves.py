"""The calls on pages run on the CPU, wave by wave: the plain reference's tables, counts and
contents whichever wave of a workgroup runs first, also with numbers out of range, and
nothing written outside the buffers."""
import ctypes

import numpy as np
import pytest

from tests import emu_util
from tests import pages_util as P

_WRAPPERS = """
namespace clsa {
hipError_t launch_zero_u32(uint32_t *p, size_t n, hipStream_t) { memset(p, 0, 4 * n); return hipSuccess; }
}
static clsa::Geometry geometry(int batch, int n_q, int max_len, int shift, int cols) {
    return clsa::Geometry{batch, n_q, batch * n_q, max_len, shift, cols, 1, 0, 8, 8, 1, 1.0f};
}
extern "C" uint32_t emu_bits() { const uint32_t v = clsa::g_device_error; clsa::g_device_error = 0; return v; }
extern "C" int emu_fork(int batch, int cols, int pages, const int32_t *parent, int32_t *table,
                        int32_t *lens, int32_t *refs, int order) {
    emu::wave_order = order;
    return clsa::launch_pages_fork(geometry(batch, 1, cols * 16, 4, cols), pages, parent, table, lens, refs, nullptr);
}
extern "C" size_t emu_reserve_ws(int batch, int n_q, int max_len, int shift, int cols) {
    return clsa::reserve_ws_ints(geometry(batch, n_q, max_len, shift, cols));
}
extern "C" int emu_reserve(int batch, int n_q, int max_len, int shift, int cols, int pages, int tensors,
                           const clsa::PagedTensor *t, const int32_t *start, const int32_t *count,
                           int32_t *table, int32_t *refs, int32_t *missing, int32_t *ws, int order) {
    emu::wave_order = order;
    return clsa::launch_pages_reserve(geometry(batch, n_q, max_len, shift, cols), pages, tensors, t, start,
                                      count, table, refs, missing, ws, nullptr);
}
extern "C" size_t emu_compact_ws(int pages) { return clsa::compact_ws_ints(pages); }
extern "C" int emu_compact(int batch, int cols, int pages, int tensors, const clsa::PagedTensor *t,
                           int32_t *table, int32_t *refs, int32_t *bound, int32_t *ws, int order) {
    emu::wave_order = order;
    return clsa::launch_pages_compact(geometry(batch, 1, cols * 16, 4, cols), pages, tensors, t, table, refs,
                                      bound, ws, nullptr);
}
extern "C" int emu_copy(int pages, int tensors, const clsa::PagedTensor *t, int n, const int32_t *src,
                        const int32_t *dst) {
    return clsa::launch_pages_copy(pages, tensors, t, n, src, dst, nullptr);
}
"""
APPEND, PAGES = 4, 16


@pytest.fixture(scope="module")
def emu(tmp_path_factory):
    lib = emu_util.build(str(tmp_path_factory.mktemp("emu")), "pages.hip", _WRAPPERS)
    lib.emu_reserve_ws.restype = lib.emu_compact_ws.restype = ctypes.c_size_t
    return lib


class Paged(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("page_bytes", ctypes.c_int64)]


class Guarded:
    """An array between guards that must stay as they are."""

    def __init__(self, x):
        x = np.ascontiguousarray(x)
        self.raw = np.full(x.nbytes + 2048, 0xA5, np.uint8)
        self.lo = 512 + (-(self.raw.ctypes.data + 512)) % 256
        self.n = x.nbytes
        self.x = self.raw[self.lo:self.lo + x.nbytes].view(x.dtype).reshape(x.shape)
        self.x[...] = x

    @property
    def p(self):
        return ctypes.c_void_p(self.x.ctypes.data)

    def intact(self):
        return bool((self.raw[:self.lo] == 0xA5).all() and (self.raw[self.lo + self.n:] == 0xA5).all())


def _tensors(rng, pages, widths=(16, 64, 20, 9000)):
    """Tensors with pages of several widths in bytes; the last is longer than a copying piece."""
    ts = [Guarded(rng.integers(0, 256, (pages, w), dtype=np.uint8)) for w in widths]
    arr = (Paged * len(ts))(*[Paged(t.x.ctypes.data, t.x.shape[1]) for t in ts])
    return ts, arr


def _moved(before, moves):
    out = [b.copy() for b in before]
    for o, b in zip(out, before):
        for a, z in moves:
            o[z] = b[a]
    return out


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("batch,cols,bad", [(1, 1, 0), (7, 5, 0), (40, 70, 0), (300, 3, 0), (9, 66, 0.1)])
def test_fork(emu, batch, cols, bad, order):
    rng = np.random.default_rng(batch * 100 + cols)
    pages = batch * cols + 3
    table, refs = P.state(rng, batch, cols, pages, bad=bad, pinned=2)
    lens = rng.integers(0, cols * 16, batch).astype(np.int32)
    parent = np.where(rng.random(batch) < 0.3, np.arange(batch), rng.integers(-1, batch, batch)).astype(np.int32)
    if bad:
        parent[rng.integers(0, batch, 2)] = [batch, -2]
    want = P.fork(parent, table, lens, refs)
    g = [Guarded(x) for x in (table, lens, refs)]
    par = Guarded(parent)
    assert emu.emu_fork(batch, cols, pages, par.p, *(x.p for x in g), order) == 0
    for x, w in zip(g, want):
        assert np.array_equal(x.x, w) and x.intact()
    assert emu.emu_bits() == (PAGES if want[3] else 0)


def test_fork_of_entries_below_none(emu):
    """A negative entry other than -1 is no page, and is reported when its slot changes hands."""
    table = np.array([[3, -5], [1, -1]], np.int32)
    refs = P.holders(table, 6)
    for parent, bits in (([0, 1], 0), ([0, 0], PAGES), ([-1, 1], PAGES)):
        parent = np.array(parent, np.int32)
        want = P.fork(parent, table, np.array([20, 5], np.int32), refs)
        g = [Guarded(x) for x in (table, np.array([20, 5], np.int32), refs)]
        assert emu.emu_fork(2, 2, 6, Guarded(parent).p, *(x.p for x in g), 0) == 0
        assert all(np.array_equal(x.x, w) for x, w in zip(g, want)) and emu.emu_bits() == bits


def _reserve(emu, rng, table, refs, start, count, n_q, page, order, tensors=True, max_len=None):
    batch, cols = table.shape
    max_len = cols * page if max_len is None else max_len
    pages = len(refs)
    ts, arr = _tensors(rng, pages) if tensors else ([], None)
    before = [t.x.copy() for t in ts]
    shift = page.bit_length() - 1
    g = [Guarded(table), Guarded(refs), Guarded(np.full(1, 77, np.int32))]
    ws = Guarded(np.full(emu.emu_reserve_ws(batch, n_q, max_len, shift, cols), -1, np.int32))
    s, c = Guarded(np.asarray(start, np.int32)), Guarded(np.asarray(count, np.int32))
    assert emu.emu_reserve(batch, n_q, max_len, shift, cols, pages, len(ts), arr, s.p, c.p, *(x.p for x in g),
                           ws.p, order) == 0
    t, r, copies, missing = P.reserve(s.x, c.x, table, refs, n_q, page, max_len)
    assert np.array_equal(g[0].x, t) and np.array_equal(g[1].x, r) and int(g[2].x[0]) == missing
    for x, w in zip(ts, _moved(before, copies)):
        assert np.array_equal(x.x, w)
    assert all(x.intact() for x in [*g, *ts, ws])
    bits = emu.emu_bits()
    odd = any(n < 0 or n > n_q or not 0 <= a <= max_len or n > max_len - a for a, n in zip(s.x.tolist(), c.x.tolist()))
    assert bool(bits & APPEND) == odd
    return bits, copies, missing


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("batch,cols,n_q,spare", [(1, 4, 1, 9), (5, 6, 1, 20), (33, 9, 40, 200), (1100, 3, 1, 1200),
                                                  (20, 8, 100, 6000), (17, 6, 3, 4), (700, 4, 1, 900),
                                                  (400, 6, 20, 9000), (400, 6, 20, 10)])
def test_reserve(emu, batch, cols, n_q, spare, order):
    rng = np.random.default_rng(batch + cols + n_q)
    pages = batch * cols + spare
    table, refs = P.state(rng, batch, cols, pages, shared=0.7, pinned=1)
    page = 16
    most = cols * page
    start = rng.integers(0, most + 1, batch)
    count = np.minimum(rng.integers(0, n_q + 1, batch), most - start)
    bits, _, missing = _reserve(emu, rng, table, refs, start, count, n_q, page, order)
    assert bool(bits & PAGES) == bool(missing)


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("batch", [150, 603, 1500])
def test_reserve_all_holders_write(emu, batch, order):
    """Every holder of a page writes: all but the last get copies, also across waves."""
    rng = np.random.default_rng(5)
    table = np.full((batch, 2), -1, np.int32)
    table[:, 0] = np.arange(batch) % 3 + 400
    refs = P.holders(table, 450 + batch)
    _, copies, missing = _reserve(emu, rng, table, refs, [3] * batch, [1] * batch, 1, 16, order)
    assert len(copies) == batch - 3 and not missing
    # one holder of each page does not write: every other one gets a copy
    count = np.ones(batch, np.int32)
    count[[10, 80, batch - 3]] = 0
    _reserve(emu, rng, table, refs, [3] * batch, count, 1, 16, order)
    # the page of 400 is held from elsewhere too
    refs[400] += 1
    _, copies, _ = _reserve(emu, rng, table, refs, [3] * batch, [1] * batch, 1, 16, order)
    assert len(copies) == batch - 2


@pytest.mark.parametrize("order", [0, 1])
def test_reserve_full_pool(emu, order):
    """Too few free pages: nothing changes, and the call says how many lack."""
    rng = np.random.default_rng(8)
    table = np.full((70, 3), -1, np.int32)
    table[:, 0] = np.arange(70) // 2
    refs = P.holders(table, 60)
    bits, copies, missing = _reserve(emu, rng, table, refs, [8] * 70, [20] * 70, 32, 16, order)
    assert bits & PAGES and not copies and missing == 70 // 2 + 70 - 25
    assert _reserve(emu, rng, table, refs, [8] * 70, [0] * 70, 32, 16, order)[2] == 0
    # exactly enough: 35 copies
    refs2 = P.holders(table, 70)
    assert _reserve(emu, rng, table, refs2, [8] * 70, [1] * 70, 32, 16, order)[2] == 0


@pytest.mark.parametrize("order", [0, 1])
def test_reserve_out_of_range(emu, order):
    rng = np.random.default_rng(3)
    table, refs = P.state(rng, 12, 5, 90, bad=0.2)
    most = 75  # the last page is not whole
    table[11, 4] = 91  # an entry that the last sequence's tokens reach
    refs = P.holders(table, 90)
    start = [0, -1, 76, 75, 74, 70, 2 ** 31 - 1, -2 ** 31, 10, 10, 33, 64]
    count = [-3, 4, 4, 1, 5, 99, 1, 1, 2 ** 31 - 1, -2 ** 31, 16, 11]
    bits, _, _ = _reserve(emu, rng, table, refs, start, count, 16, 16, order, max_len=most)
    assert bits & APPEND and bits & PAGES
    # counts that do not match the table: any result, inside the buffers
    for seed in range(4):
        r = rng.integers(-3, 4, 90).astype(np.int32)
        ts, arr = _tensors(rng, 90)
        g = [Guarded(table), Guarded(r), Guarded(np.zeros(1, np.int32))]
        ws = Guarded(np.full(emu.emu_reserve_ws(12, 16, 80, 4, 5), -1, np.int32))
        s, c = Guarded(np.arange(12, dtype=np.int32) * 6), Guarded(np.full(12, 9, np.int32))
        assert emu.emu_reserve(12, 16, 80, 4, 5, 90, len(ts), arr, s.p, c.p, *(x.p for x in g), ws.p, order) == 0
        assert all(x.intact() for x in [*g, *ts, ws])
    emu.emu_bits()


@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("batch,cols,pages,pinned,bad", [(1, 1, 1, 0, 0), (6, 5, 31, 0, 0), (30, 9, 500, 9, 0),
                                                         (4, 3, 2100, 0, 0), (8, 8, 64, 3, 0.1), (5, 900, 9001, 5, 0),
                                                         (5, 9, 8200, 2, 0.1)])
def test_compact(emu, batch, cols, pages, pinned, bad, order):
    rng = np.random.default_rng(pages)
    table, refs = P.state(rng, batch, cols, pages, shared=0.6, pinned=pinned, bad=bad)
    ts, arr = _tensors(rng, pages)
    before = [t.x.copy() for t in ts]
    g = [Guarded(table), Guarded(refs), Guarded(np.full(1, 77, np.int32))]
    ws = Guarded(np.full(emu.emu_compact_ws(pages), -1, np.int32))
    assert emu.emu_compact(batch, cols, pages, len(ts), arr, *(x.p for x in g), ws.p, order) == 0
    t, r, moves, bound = P.compact(table, refs)
    assert np.array_equal(g[0].x, t) and np.array_equal(g[1].x, r) and int(g[2].x[0]) == bound
    for x, w in zip(ts, _moved(before, moves)):
        assert np.array_equal(x.x, w)
    assert all(x.intact() for x in [*g, *ts, ws])
    assert emu.emu_bits() == (PAGES if bad else 0)


def test_compact_counts_that_do_not_match(emu):
    rng = np.random.default_rng(2)
    for seed in range(4):
        table, _ = P.state(rng, 6, 5, 40, bad=0.1)
        g = [Guarded(table), Guarded(rng.integers(-3, 4, 40).astype(np.int32)), Guarded(np.zeros(1, np.int32))]
        ts, arr = _tensors(rng, 40)
        ws = Guarded(np.full(emu.emu_compact_ws(40), -1, np.int32))
        assert emu.emu_compact(6, 5, 40, len(ts), arr, *(x.p for x in g), ws.p, 0) == 0
        assert all(x.intact() for x in [*g, *ts, ws])
    emu.emu_bits()


def test_copy(emu):
    rng = np.random.default_rng(4)
    ts, arr = _tensors(rng, 50)
    before = [t.x.copy() for t in ts]
    src = Guarded(np.array([0, -1, 49, 7, 7, 50, 3, -2, 5], np.int32))
    dst = Guarded(np.array([10, 11, 12, 13, 14, 15, 50, 16, -1], np.int32))
    assert emu.emu_copy(50, len(ts), arr, 9, src.p, dst.p) == 0
    for x, w in zip(ts, _moved(before, [(0, 10), (49, 12), (7, 13), (7, 14)])):
        assert np.array_equal(x.x, w) and x.intact()
    assert emu.emu_bits() == PAGES
