"""The residual norm and its backward pass on the GPU against the formulas in 64 bits.

Bounds: s is bf16(fp32(x + residual)), rounded the same way here: equal bits.  rstd: one
rounding to fp32, 2^-24 (a subnormal one: half its step).  y: three fp32 roundings and the one to
bf16, 2^-8.  The bytes are those of the same fp32 products over the group's scale, byte by
byte."""
import numpy as np
import pytest

from paper_2606_06467_amd import inputs
from tests import cache8_util as C
from tests import gpu_util as U

pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24
EPS = 1e-6
FORMS = [(1, 8), (1, 2560), (3, 72), (5, 1000), (77, 8200), (2, 16384), (256, 16), (257, 16), (320, 2560), (321, 2560), (1500, 520), (1030, 2560), (1100, 4096),
         (1029, 4104), (2050, 8), (1027, 3592),
         (768, 5120), (769, 1000), (600, 8), (1030, 1544), (4100, 2080), (1100, 8008), (17000, 512)]


def f32(bits):
    return inputs.f32_from_bf16_bits(bits)


def round_bf16(x):
    """fp32 -> bf16 bits, nearest even (finite values)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def _inputs(rows, d, seed, scale=1.0):
    x = inputs.normal_bf16(seed, (rows, d), scale)
    r = inputs.normal_bf16(seed + 1, (rows, d), 3 * scale)
    w = round_bf16(1 + 0.3 * f32(inputs.normal_bf16(seed + 2, (d,), 1.0)))
    return x, r, w


def _run(x, r, w, group, rows, d, y=True, eps=EPS, alias=False, stream=None, want_sum=True):
    import torch
    from paper_2606_06467_amd import binding as B
    sh = B.make_shape(1, rows, 1, 1)
    X, W = B.bf16_from_bits(x), B.bf16_from_bits(w)
    R = None if r is None else B.bf16_from_bits(r)
    s = R if alias else torch.full((rows, d), 9.0, dtype=torch.bfloat16, device="cuda") if want_sum else None
    o = X if alias else torch.full((rows, d), 9.0, dtype=torch.bfloat16, device="cuda") if y else None
    y8 = sc = None
    if group:
        y8 = torch.full((rows, d), 0x55, dtype=torch.uint8, device="cuda")
        sc = torch.full((rows, -(-d // group)), 7.0, device="cuda")
    rstd = torch.full((rows,), 7.0, device="cuda")
    B.clsa_residual_norm(sh, d, eps, X, R, W, s, o, y8, sc, rstd, stream, group=group or 128)
    torch.cuda.synchronize()
    return dict(s=None if s is None else B.bits_from_bf16(s), y=None if o is None else B.bits_from_bf16(o),
                y8=None if y8 is None else y8.cpu().numpy(), scale=None if sc is None else sc.cpu().numpy(),
                rstd=rstd.cpu().numpy())


def _scales(y, group):
    """Scales of fp32 values by group, and the largest finite magnitudes that they come from."""
    rows, d = y.shape
    n = -(-d // group)
    a = np.zeros((rows, n * group), np.float64)
    a[:, :d] = np.where(np.isfinite(y), np.abs(y), 0)
    top = np.minimum(a.reshape(rows, n, group).max(2), C.TOP)
    with np.errstate(divide="ignore"):
        e = np.maximum(np.ceil(np.log2(top / 448)), -100)
    e = np.where(448 * 2.0 ** (e - 1) >= top, e - 1, e)       # where log2 rounded up past a whole number
    e = np.where(448 * 2.0 ** e < top, e + 1, e)
    return 2.0 ** np.maximum(e, -100)


def _check(got, x, r, w, group, eps=EPS):
    s = x if r is None else round_bf16(f32(x) + f32(r))
    if got["s"] is not None:
        assert np.array_equal(got["s"], s)
    v = f32(s).astype(np.float64)
    rstd = 1 / np.sqrt((v * v).mean(1) + eps)
    assert np.all(np.abs(got["rstd"] - rstd) <= rstd * U24 * (1 + 1e-6) + 2.0 ** -150)
    y32 = (f32(s) * got["rstd"][:, None]) * f32(w)
    if got["y"] is not None:
        y = v * rstd[:, None] * f32(w)
        err = np.abs(f32(got["y"]) - y)
        assert np.all(err <= np.abs(y) * (2.0 ** -8 + 4 * U24) + 2.0 ** -133)
    if got["y8"] is not None:
        sc = _scales(y32, group)
        assert np.array_equal(got["scale"], sc.astype(np.float32))
        each = np.repeat(sc, group, 1)[:, :y32.shape[1]]
        z = np.where(np.isfinite(y32), np.clip(y32.astype(np.float64), -C.TOP, C.TOP), np.nan)
        assert C.same_bytes(got["y8"], C.encode(z / each))


@pytest.mark.parametrize("rows,d", FORMS)
@pytest.mark.parametrize("group", [0, 32, 64, 128, "row"])
def test_norm(rows, d, group):
    x, r, w = _inputs(rows, d, 900 + rows + d)
    group = d if group == "row" else group
    got = _run(x, r, w, group, rows, d)
    _check(got, x, r, w, group)
    if group:  # bytes alone, and without a residual
        one = _run(x, None, w, group, rows, d, y=False, want_sum=False)
        _check(one, x, None, w, group)


@pytest.mark.parametrize("rows,d", [(4, 2560), (1100, 2560), (3, 12288)])
def test_norm_in_place(rows, d):
    x, r, w = _inputs(rows, d, 31)
    a, b = _run(x, r, w, 64, rows, d), _run(x, r, w, 64, rows, d, alias=True)
    for k in a:
        assert np.array_equal(a[k], b[k]), k


@pytest.mark.parametrize("rows", [9, 1032])
@pytest.mark.parametrize("group", [32, "row"])
def test_norm_odd_values(rows, group):
    """Rows of zeros, of the largest and least values, with infinities and NaN: their own rows only."""
    d = 264
    group = d if group == "row" else group
    x, r, w = _inputs(rows, d, 77)
    r[:] = 0
    x[0] = 0                                    # zeros
    x[1] = 0x7F7F                               # the largest bf16: squares past fp32
    x[2] = 0x0001                               # the least subnormal
    x[3, 40] = 0x7F80                           # an infinity
    x[4, 41] = 0x7FC1                           # a NaN
    x[5] = 0x7F7F
    r[5] = 0x7F7F                               # a sum past bf16: infinities
    x[6, 7], r[6, 7] = 0x7F80, 0xFF80           # inf - inf
    x[7, 3] = 0x7F00                            # one value that outweighs its row
    got = _run(x, r, w, group, rows, d)
    with np.errstate(invalid="ignore", over="ignore"):
        s32 = f32(x) + f32(r)
        top = f32(np.array([0x7F7F], np.uint16))[0]
        s = np.where(np.isnan(s32), np.float32(np.nan), np.where(np.abs(s32) > top, np.copysign(np.float32(np.inf), s32), s32))
        v = s.astype(np.float64)
        rstd = 1 / np.sqrt((v * v).mean(1) + EPS)
    plain = [i for i in range(rows) if i not in (3, 4, 5, 6)]
    _check({k: None if a is None else a[plain] for k, a in got.items()}, x[plain], r[plain], w, group)
    assert got["rstd"][3] == 0 and got["rstd"][5] == 0 and np.isnan(got["rstd"][[4, 6]]).all()
    assert np.all(f32(got["s"][5]) == np.inf) and np.isnan(f32(got["s"][6])[7]) and np.isnan(f32(got["s"][4])[41])
    with np.errstate(invalid="ignore"):
        y = v * rstd[:, None] * f32(w)
    for i in (3, 4, 5, 6):
        g = f32(got["y"][i])
        assert np.array_equal(np.isnan(g), np.isnan(y[i])) and np.all(g[~np.isnan(g)] == 0)
        assert np.array_equal((got["y8"][i] & 0x7F) == 0x7F, np.isnan(y[i]))
    assert np.all(got["scale"][0] == 2.0 ** -100) and not (got["y8"][0] & 0x7F).any()


def _grad(s, rstd, w, dy, ds, rows, d, alias=False, poison=None, stream=None):
    import torch
    from paper_2606_06467_amd import binding as B
    sh = B.make_shape(rows, 1, 1, 1)
    S, W, DY = (B.bf16_from_bits(v) for v in (s, w, dy))
    DS = None if ds is None else B.bf16_from_bits(ds)
    dx = (DY if ds is None else DS) if alias else torch.full((rows, d), 9.0, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((d,), 7.0, device="cuda")
    ws = B.workspace(sh, B.CLSA_OP_NORM_GRAD, d)
    if poison is not None:
        ws.fill_(poison)
    B.clsa_residual_norm_grad(sh, d, S, torch.from_numpy(rstd).cuda(), W, DY, DS, dx, dw, ws, stream)
    torch.cuda.synchronize()
    return B.bits_from_bf16(dx), dw.cpu().numpy()


def _grad_inputs(rows, d, seed):
    s, _, w = _inputs(rows, d, seed)
    v = f32(s).astype(np.float64)
    rstd = (1 / np.sqrt((v * v).mean(1) + EPS)).astype(np.float32)
    return s, rstd, w, inputs.normal_bf16(seed + 5, (rows, d), 1e-2), inputs.normal_bf16(seed + 6, (rows, d), 1e-2)


def _check_grad(got, s, rstd, w, dy, ds):
    """fp32 sums of d (and of rows) terms: at most n u times the sum of magnitudes (each term
    has up to three roundings, each result a few more), then the rounding to bf16."""
    rows, d = s.shape
    xh, g, y = f32(s).astype(np.float64) * rstd[:, None], f32(dy) * f32(w).astype(np.float64), f32(dy).astype(np.float64)
    r = rstd[:, None].astype(np.float64)
    c, c_abs = (g * xh).mean(1, keepdims=True), np.abs(g * xh).mean(1, keepdims=True)
    ref = r * (g - xh * c)
    if ds is not None:
        ref = ref + f32(ds)
    tol = np.abs(ref) * 2.0 ** -8 + r * U24 * ((d + 4) * c_abs * np.abs(xh) + 6 * (np.abs(g) + np.abs(xh * c))) + 2.0 ** -133
    err = np.abs(f32(got[0]) - ref)
    assert np.all(err <= tol * (1 + 2.0 ** -8)), float((err / tol).max())
    dw, mag = (y * xh).sum(0), np.abs(y * xh).sum(0)
    assert np.all(np.abs(got[1] - dw) <= (rows + 4) * U24 * mag + 1e-40)


@pytest.mark.parametrize("rows,d", FORMS + [(1100, 1200), (8200, 1024), (5600, 1504), (4200, 2048)])
def test_norm_grad(rows, d):
    s, rstd, w, dy, ds = _grad_inputs(rows, d, 70 + rows + d)
    got = _grad(s, rstd, w, dy, ds, rows, d)
    _check_grad(got, s, rstd, w, dy, ds)
    _check_grad(_grad(s, rstd, w, dy, None, rows, d), s, rstd, w, dy, None)
    _check_grad(_grad(s, rstd, w, dy, None, rows, d, alias=True), s, rstd, w, dy, None)  # in dy's place
    # the same bits again, whatever the workspace holds, and in place
    for again in (_grad(s, rstd, w, dy, ds, rows, d, poison=0xFF), _grad(s, rstd, w, dy, ds, rows, d, alias=True)):
        assert np.array_equal(again[0], got[0]) and np.array_equal(again[1], got[1])


def test_norm_grad_against_differences():
    """Central differences of sum(dy y) in 64 bits, with respect to s and the weight."""
    rows, d = 3, 24
    s, rstd, w, dy, _ = _grad_inputs(rows, d, 4)
    dx, dw = _grad(s, rstd, w, dy, None, rows, d)
    v, wt, g = f32(s).astype(np.float64), f32(w).astype(np.float64), f32(dy).astype(np.float64)

    def loss(v, wt):
        return (g * v / np.sqrt((v * v).mean(1, keepdims=True) + EPS) * wt).sum()

    h = 1e-5
    for i in range(rows):
        for j in range(d):
            e = np.zeros_like(v)
            e[i, j] = h
            num = (loss(v + e, wt) - loss(v - e, wt)) / (2 * h)
            # bf16 half a step, 2^-8; the difference quotient: h^2 of the third derivative, 1e-8
            assert abs(f32(dx[i:i + 1, j])[0] - num) <= 2.0 ** -8 * abs(num) + 1e-7
    for j in range(d):
        e = np.zeros_like(wt)
        e[j] = h
        assert abs(dw[j] - (loss(v, wt + e) - loss(v, wt - e)) / (2 * h)) <= 1e-7


def test_norm_of_offsets_past_32_bits():
    """2^22 - 1 rows of 1032 values: the last rows like the same rows alone."""
    import torch
    from paper_2606_06467_amd import binding as B
    rows, d, n = (1 << 22) - 1, 1032, 5
    x = torch.full((rows, d), 0.5, dtype=torch.bfloat16, device="cuda")
    end = B.bf16_from_bits(inputs.normal_bf16(1, (n, d), 1.0))
    x[-n:] = end
    w = B.bf16_from_bits(inputs.normal_bf16(2, (d,), 1.0))
    y, few = torch.empty_like(x), torch.empty_like(end)
    rstd, dw, dw1 = torch.empty(rows, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    sh, one = B.make_shape(rows, 1, 1, 1), B.make_shape(n, 1, 1, 1)
    B.clsa_residual_norm(sh, d, EPS, x, None, w, y=y, rstd=rstd)
    B.clsa_residual_norm(one, d, EPS, end, None, w, y=few)
    assert torch.equal(y[-n:].view(torch.int16), few.view(torch.int16))
    # the gradient in place of y, from dy = x
    B.clsa_residual_norm_grad(sh, d, x, rstd, w, x, None, y, dw, B.workspace(sh, B.CLSA_OP_NORM_GRAD, d))
    B.clsa_residual_norm_grad(one, d, end, rstd[-n:].contiguous(), w, end, None, few, dw1,
                              B.workspace(one, B.CLSA_OP_NORM_GRAD, d))
    assert torch.allclose(y[-n:].float(), few.float(), rtol=2 ** -7, atol=1e-6)  # sums of d in another order
    # dw = sum of x^2 rstd: rows - n equal terms of 0.25 / sqrt(0.25 + EPS), summed in fp32 by few
    # chains of rows / 2048 at most: that many roundings
    want = (rows - n) * 0.25 / (0.25 + EPS) ** 0.5
    assert torch.all((dw - want).abs() <= want * (rows / 512 + 300) * U24 + dw1.abs())


def test_norm_on_a_stream_and_replayed():
    """Captured on another stream: every replay gives the eager bits, with eager work between."""
    import torch
    from paper_2606_06467_amd import binding as B
    rows, d = 1100, 2560
    x, r, w = _inputs(rows, d, 8)
    sh = B.make_shape(rows, 1, 1, 1)
    X, R, W, DY = (B.bf16_from_bits(v) for v in (x, r, w, inputs.normal_bf16(3, (rows, d), 1e-2)))
    s, y, dx = (torch.empty((rows, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    y8 = torch.empty((rows, d), dtype=torch.uint8, device="cuda")
    sc, rstd, dw = torch.empty((rows, 20), device="cuda"), torch.empty(rows, device="cuda"), torch.empty(d, device="cuda")
    ws = B.workspace(sh, B.CLSA_OP_NORM_GRAD, d)
    outs = (s, y, y8, sc, rstd, dx, dw)

    def step(stream=None):
        B.clsa_residual_norm(sh, d, EPS, X, R, W, s, y, y8, sc, rstd, stream)
        B.clsa_residual_norm_grad(sh, d, s, rstd, W, DY, None, dx, dw, ws, stream)

    step()
    torch.cuda.synchronize()
    ref = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in outs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outs, ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outs, ref))
        step()
        torch.cuda.synchronize()


@pytest.mark.parametrize("rows,d", [(1, 8), (3, 72), (77, 1000), (256, 2560), (300, 512), (768, 520), (2, 16384), (769, 520), (1500, 520), (1030, 4104)])
@pytest.mark.parametrize("place", ["dy", "s"])
def test_norm_grad_in_place_has_the_same_bits(rows, d, place):
    """dx in the place of dy or of s: the bits of dx and dweight on their own, with and without dsum."""
    import torch
    from paper_2606_06467_amd import binding as B
    s, rstd, w, dy, ds = _grad_inputs(rows, d, 40 + rows + d)
    sh, R, W = B.make_shape(rows, 1, 1, 1), torch.from_numpy(rstd).cuda(), B.bf16_from_bits(w)
    ws = B.workspace(sh, B.CLSA_OP_NORM_GRAD, d)
    for more in (None, B.bf16_from_bits(ds)):
        want = _grad(s, rstd, w, dy, None if more is None else ds, rows, d)
        t = dict(s=B.bf16_from_bits(s), dy=B.bf16_from_bits(dy))
        dw = torch.full((d,), 7.0, device="cuda")
        B.clsa_residual_norm_grad(sh, d, t["s"], R, W, t["dy"], more, t[place], dw, ws)
        torch.cuda.synchronize()
        assert np.array_equal(B.bits_from_bf16(t[place]), want[0])
        assert np.array_equal(dw.cpu().numpy().view(np.uint32), want[1].view(np.uint32))
