"""Host-only checks of the norm, adapter and page entry points: what they refuse (before
anything is enqueued), and the workspaces that they ask for."""
import ctypes

import pytest
import torch

from paper_2606_06467_amd import binding as B

# Fake, aligned, never-dereferenced device addresses: every call below must be rejected.
A = ctypes.c_void_p(0x10000)
MIS = ctypes.c_void_p(0x10002)
BIG = 1 << 40


def _shape(**kw):
    base = dict(batch=2, n_q=1, max_len=1024, top_k=1)
    base.update(kw)
    return B.make_shape(**base)


def _paged(**kw):
    return _shape(**{**dict(page_size=64, max_pages=16), **kw})


def _norm(sh, d=512, eps=1e-6, group=128, x=A, res=A, w=A, s=A, y=A, y8=A, ys=A, rstd=A):
    return B.lib().clsa_residual_norm(ctypes.byref(sh), d, eps, group, x, res, w, s, y, y8, ys, rstd, None)


def _grad(sh, d=512, s=A, rstd=A, w=A, dy=A, ds=A, dx=A, dw=A, ws=None, wsb=0):
    return B.lib().clsa_residual_norm_grad(ctypes.byref(sh), d, s, rstd, w, dy, ds, dx, dw, ws, wsb, None)


def _adapted(sh, d=512, n=2, rank=16, h=A, w=A, a=A, b=A, al=A, ad=A, pos=A, pt=None, q=A, ki=A, k=A, v=A, ws=None,
             wsb=0):
    return B.lib().clsa_project_append_adapted(ctypes.byref(sh), d, n, rank, h, w, a, b, al, ad, pos, pt, q, ki, k,
                                               v, ws, wsb, None)


def _adapted8(sh, block=64, d=512, n=2, rank=16, h=A, w=A, a=A, b=A, al=A, ad=A, start=A, count=A, pt=None, q=A,
              ki=A, k8=A, v8=A, ks=A, vs=A, ws=None, wsb=0):
    return B.lib().clsa_project_append8_adapted(ctypes.byref(sh), block, d, n, rank, h, w, a, b, al, ad, start,
                                                count, pt, q, ki, k8, v8, ks, vs, ws, wsb, None)


def _tensors(*pairs):
    return (B.ClsaPaged * max(1, len(pairs)))(*[B.ClsaPaged(p, n) for p, n in pairs])


ONE = _tensors((0x10000, 64))


def _fork(sh, pages=10, par=A, pt=A, sl=A, refs=A):
    return B.lib().clsa_pages_fork(ctypes.byref(sh), pages, par, pt, sl, refs, None)


def _reserve(sh, pages=10, n=1, t=ONE, start=A, count=A, pt=A, refs=A, miss=A, ws=None, wsb=0):
    return B.lib().clsa_pages_reserve(ctypes.byref(sh), pages, n, t, start, count, pt, refs, miss, ws, wsb, None)


def _compact(sh, pages=10, n=1, t=ONE, pt=A, refs=A, bound=A, ws=None, wsb=0):
    return B.lib().clsa_pages_compact(ctypes.byref(sh), pages, n, t, pt, refs, bound, ws, wsb, None)


def _copy(pages=10, n=1, t=ONE, m=3, src=A, dst=A):
    return B.lib().clsa_pages_copy(pages, n, t, m, src, dst, None)


def test_norm_refusals():
    sh = _shape()
    assert _norm(_shape(batch=0)) == -1 and _norm(_shape(n_q=0)) == -1
    assert B.lib().clsa_residual_norm(None, 512, 1e-6, 128, A, A, A, A, A, A, A, A, None) == -1
    for d, code in ((0, -1), (-8, -1), (12, -2), (16392, -2)):
        assert _norm(sh, d=d) == code and _grad(sh, d=d) == code, d
    assert _norm(_shape(batch=1 << 12, n_q=1 << 10)) == -2   # 2^22 rows
    for eps in (0.0, -1e-6, float("nan"), float("inf"), 1e-39):
        assert _norm(sh, eps=eps) == -1, eps
    for group, code in ((0, -1), (-128, -1), (16, -2), (96, -2), (256, -2)):
        assert _norm(sh, group=group) == code, group
    for name in ("x", "w"):
        for bad in (None, MIS):
            assert _norm(sh, **{name: bad}) == -1, name
    for name in ("res", "s", "y", "y8", "ys"):
        assert _norm(sh, **{name: MIS}) == -1, name
    assert _norm(sh, rstd=ctypes.c_void_p(0x10001)) == -1
    assert _norm(sh, y8=None) == -1 and _norm(sh, ys=None) == -1      # one of them alone
    assert _norm(sh, y=None, y8=None, ys=None) == -1                  # no result


def test_norm_grad_refusals():
    sh = _shape()
    need = B.clsa_workspace_bytes(sh, B.CLSA_OP_NORM_GRAD, 512)
    assert need >= 512 * 4 and B.clsa_workspace_bytes(sh, B.CLSA_OP_NORM_GRAD, 12) == 0
    for name in ("s", "rstd", "w", "dy", "dx", "dw"):
        assert _grad(sh, ws=A, wsb=need, **{name: None}) == -1, name
    assert _grad(sh, ws=A, wsb=need, ds=MIS) == -1
    assert _grad(sh) == -3 and _grad(sh, ws=A, wsb=need - 1) == -3
    assert _grad(sh, ws=ctypes.c_void_p(0x10010), wsb=BIG) == -3


@pytest.mark.parametrize("call,op", [(_adapted, B.CLSA_OP_ADAPTED), (_adapted8, B.CLSA_OP_ADAPTED8)])
def test_adapter_refusals(call, op):
    sh = _shape()
    ok = dict(ws=A, wsb=BIG)
    for n, rank, code in ((0, 16, -1), (-1, 16, -1), (2, 0, -1), (2, -8, -1), (2, 4, -2), (2, 20, -2), (2, 136, -2)):
        assert call(sh, n=n, rank=rank, **ok) == code, (n, rank)
    for d, code in ((0, -1), (500, -2), (8704, -2)):
        assert call(sh, d=d, **ok) == code, d
    for name in ("h", "w", "a", "b", "al", "ad", "q", "ki"):
        assert call(sh, **{name: None}, **ok) == -1, name
    for name in ("h", "w", "a", "b", "q", "ki"):
        assert call(sh, **{name: MIS}, **ok) == -1, name
    for rank in (8, 16, 128):
        need = B.clsa_workspace_bytes(sh, op, rank)
        assert need >= 2 * rank * 4
        assert call(sh, rank=rank) == -3 and call(sh, rank=rank, ws=A, wsb=need - 1) == -3
    assert B.clsa_workspace_bytes(sh, op, 12) == 0 and B.clsa_workspace_bytes(sh, op, 0) == 0
    assert call(_shape(head_dim=64), **ok) == -2 and call(_paged(), **ok) == -1  # no page table
    assert call(_shape(batch=0), **ok) == -1


def test_adapter8_blocks():
    for block, code in ((0, -1), (48, -2), (256, -2)):
        assert _adapted8(_shape(), block=block, ws=A, wsb=BIG) == code
    assert _adapted8(_paged(page_size=32, max_pages=32), block=64, pt=A, ws=A, wsb=BIG) == -2


@pytest.mark.parametrize("call", [_fork, _reserve, _compact])
def test_page_shapes(call):
    more = {} if call is _fork else dict(ws=A, wsb=BIG)
    assert call(_shape(), **more) == -1                       # contiguous
    assert call(_paged(max_pages=15), **more) == -1           # columns short of max_len
    assert call(_paged(page_size=48, max_len=960, max_pages=20), **more) == -1
    assert call(_paged(page_size=8, max_pages=128), **more) == -2
    assert call(_paged(batch=0), **more) == -1
    for pages, code in ((0, -1), (-5, -1), ((1 << 24) + 1, -2)):
        assert call(_paged(), pages=pages, **more) == code, pages
    for name in ("pt", "refs"):
        for bad in (None, ctypes.c_void_p(0x10001)):
            assert call(_paged(), **{name: bad}, **more) == -1, name


def test_page_refusals():
    sh = _paged()
    for name in ("par", "sl"):
        assert _fork(sh, **{name: None}) == -1
    assert _fork(_paged(batch=16385)) == -2
    ok = dict(ws=A, wsb=BIG)
    for name in ("start", "count", "miss"):
        assert _reserve(sh, **{name: None}, **ok) == -1, name
    assert _compact(sh, bound=None, **ok) == -1
    for call in (_reserve, _compact):
        for t, n, code in ((None, 1, -1), (ONE, -1, -1), (ONE, 17, -2), (_tensors((0, 64)), 1, -1),
                           (_tensors((0x10002, 64)), 1, -1), (_tensors((0x10000, 0)), 1, -1),
                           (_tensors((0x10000, 6)), 1, -1), (_tensors((0x10000, -4)), 1, -1),
                           (_tensors((0x10000, (1 << 30) + 4)), 1, -2)):
            assert call(sh, n=n, t=t, **ok) == code, (n, code)
    need = B.clsa_workspace_bytes(sh, B.CLSA_OP_PAGES_RESERVE)
    assert need > 0 and _reserve(sh) == -3 and _reserve(sh, ws=A, wsb=need - 1) == -3
    need = B.clsa_workspace_bytes(sh, B.CLSA_OP_PAGES_COMPACT, 10)
    assert need >= 160 and _compact(sh) == -3 and _compact(sh, ws=A, wsb=need - 1) == -3
    assert B.clsa_workspace_bytes(_shape(), B.CLSA_OP_PAGES_RESERVE) == 0
    assert B.clsa_workspace_bytes(sh, B.CLSA_OP_PAGES_COMPACT, 0) == 0
    huge = _paged(batch=1 << 16, n_q=1 << 14, max_len=1 << 14, page_size=16, max_pages=1 << 10)
    assert _reserve(huge, **ok) == -2 and B.clsa_workspace_bytes(huge, B.CLSA_OP_PAGES_RESERVE) == 0


def test_copy_refusals():
    for kw, code in ((dict(pages=0), -1), (dict(pages=(1 << 24) + 1), -2), (dict(m=-1), -1), (dict(src=None), -1),
                     (dict(dst=ctypes.c_void_p(0x10001)), -1), (dict(t=None), -1), (dict(n=17), -2)):
        assert _copy(**kw) == code, kw
    assert _copy(m=0, src=None, dst=None) == 0    # nothing to do


def test_binding_takes_gpu_tensors_only():
    x = torch.zeros((2, 512), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="x must be a GPU tensor"):
        B.clsa_residual_norm(_shape(), 512, 1e-6, x, None, x[0], y=x)
    with pytest.raises(ValueError, match="GPU tensor"):
        B.clsa_pages_fork(_paged(), i, i, i, i)
    with pytest.raises(ValueError, match=r"tensors\[0\] must be a GPU tensor"):
        B.clsa_pages_reserve(_paged(), [x], i, i, i, i, i)
    for a, b in ((x, x), (x[None], None), (x[None], x[None, :1]), (x[None], torch.zeros(2, 8, 2))):
        with pytest.raises(ValueError, match="three dimensions|one rank"):
            B.clsa_project_append_adapted(_shape(), 512, x, x, a, b, x, i, i, None, x, x, x, x)
        with pytest.raises(ValueError, match="three dimensions|one rank"):
            B.clsa_project_append8_adapted(_shape(), 64, 512, x, x, a, b, x, i, i, i, None, x, x, x, x, x, x)
    with pytest.raises(TypeError, match=r"tensors\[0\]"):
        B.clsa_pages_compact(_paged(), [None], i, i, i)


def test_binding_compares_adapters_with_the_shape():
    """Sizes that the library takes from the shape: refused before any device address is asked for."""
    sh = _shape(kv_heads=2, q_heads=2)     # 1024 features, 2 sequences
    x, i = torch.zeros((2, 512), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    ok = dict(a=(3, 8, 512), b=(3, 1024, 8), alpha=(3,), adapter=(2,))

    def call(which, **kw):
        t = {k: torch.zeros(v, dtype=torch.int32 if k == "adapter" else torch.float32 if k == "alpha" else torch.bfloat16)
             for k, v in {**ok, **kw}.items()}
        if which == 8:
            B.clsa_project_append8_adapted(sh, 64, 512, x, x, *t.values(), i, i, None, x, x, x, x, x, x)
        else:
            B.clsa_project_append_adapted(sh, 512, x, x, *t.values(), i, None, x, x, x, x)

    for which in (16, 8):
        for bad, what in ((dict(a=(3, 8, 1024)), "a must hold vectors of d_model 512"),
                          (dict(a=(3, 8, 256)), "a must hold vectors of d_model 512"),
                          (dict(b=(3, 768, 8)), "b must hold the shape's 1024 features"),
                          (dict(b=(3, 2560, 8)), "b must hold the shape's 1024 features"),
                          (dict(alpha=(2,)), "alpha must hold a factor for each of the 3"),
                          (dict(adapter=(1,)), "adapter must hold a number for each of the 2"),
                          ({}, "h must be a GPU tensor"), (dict(adapter=(9,)), "h must be a GPU tensor")):
            with pytest.raises(ValueError, match=what):
                call(which, **bad)


@pytest.mark.parametrize("eps", [3.5e38, 1e60, 1e300])
def test_norm_refuses_an_eps_past_fp32(eps):
    """As an invalid argument, before it looks at a group that it does not have."""
    assert _norm(_shape(), group=16) == -2
    assert _norm(_shape(), eps=eps, group=16) == -1
