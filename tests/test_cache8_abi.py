"""Host-only checks of the 8-bit cache and block routing entry points: what they refuse
(before anything is enqueued), their workspaces, and the tests' own e4m3 reference."""
import ctypes
import importlib.util
import types

import numpy as np
import pytest
import torch

from paper_2606_06467_amd import binding as B
from tests import cache8_util as C

# Fake, aligned, never-dereferenced device addresses: every call below must be rejected.
A = ctypes.c_void_p(0x10000)
MIS = ctypes.c_void_p(0x10002)


def _shape(**kw):
    base = dict(batch=2, n_q=1, max_len=1024, top_k=128)
    base.update(kw)
    return B.make_shape(**base)


def _append(sh, block=64, k=A, v=A, start=A, count=A, pt=None, k8=A, v8=A, ks=A, vs=A):
    return B.lib().clsa_cache_append8(ctypes.byref(sh), block, k, v, start, count, pt, k8, v8, ks, vs, None)


def _sparse(sh, block=64, q=A, k8=A, v8=A, ks=A, vs=A, pt=None, idx=A, ns=A, out=A, lse=None, ws=None,
            wsb=0):
    return B.lib().clsa_sparse_attn8(ctypes.byref(sh), block, q, k8, v8, ks, vs, pt, idx, ns, out, lse, ws,
                                     wsb, None)


def _dense(sh, block=64, q=A, k8=A, v8=A, ks=A, vs=A, pt=None, sl=A, qp=None, out=A, lse=None, ws=None,
           wsb=0):
    return B.lib().clsa_dense_attn8(ctypes.byref(sh), block, q, k8, v8, ks, vs, pt, sl, qp, out, lse, ws,
                                    wsb, None)


def _means(sh, block=64, ki=A, start=A, count=A, pt=None, m=A):
    return B.lib().clsa_block_means(ctypes.byref(sh), block, ki, start, count, pt, m, None)


def _topk(sh, block=64, q=A, m=A, pt=None, sl=A, qp=None, idx=A, ns=A, ws=None, wsb=0):
    return B.lib().clsa_block_topk(ctypes.byref(sh), block, q, m, pt, sl, qp, idx, ns, ws, wsb, None)


def _project(sh, block=64, d=512, h=A, w=A, start=A, count=A, pt=None, q=A, ki=A, k8=A, v8=A, ks=A, vs=A,
             ws=None, wsb=0):
    return B.lib().clsa_project_append8(ctypes.byref(sh), block, d, h, w, start, count, pt, q, ki, k8, v8, ks,
                                        vs, ws, wsb, None)


CALLS = [_append, _sparse, _dense, _means, _topk, _project]


@pytest.mark.parametrize("call", CALLS)
def test_blocks(call):
    for block, code in ((0, -1), (-64, -1), (8, -2), (48, -2), (256, -2)):
        assert call(_shape(), block=block) == code, block
    # a block lies inside one page
    assert call(_shape(page_size=32, max_pages=32), block=64, pt=A) == -2
    assert call(_shape(page_size=64, max_pages=16), pt=None) == -1
    assert call(_shape(page_size=64, max_pages=15), pt=A) == -1


@pytest.mark.parametrize("call", CALLS)
def test_shapes(call):
    assert call(_shape(batch=0)) == -1
    assert call(_shape(n_q=0)) == -1
    sh = _shape()
    sh.causal = 2
    assert call(sh) == -1
    assert call(_shape(top_k=8193)) in (-1, -2)
    if call in (_append, _sparse, _dense, _project):
        assert call(_shape(head_dim=64)) == -2
        assert call(_shape(q_heads=48, kv_heads=8)) == -2
        assert call(_shape(q_heads=32, kv_heads=5)) == -1
        assert call(_shape(softmax_scale=float("nan"))) == -1
        assert call(_shape(max_len=262144, q_heads=64, kv_heads=64)) == -2
    if call in (_means, _topk, _project):
        assert call(_shape(idx_dim=32)) == -2
    if call in (_dense, _topk, _means, _project):
        assert call(_shape(max_len=262145)) == -2


@pytest.mark.parametrize("call,names,align", [
    (_append, ("k", "v", "k8", "v8"), 16), (_append, ("start", "count", "ks", "vs"), 4),
    (_sparse, ("q", "k8", "v8", "out"), 16), (_sparse, ("ks", "vs", "idx", "ns"), 4),
    (_dense, ("q", "k8", "v8", "out"), 16), (_dense, ("ks", "vs", "sl"), 4),
    (_means, ("ki", "m"), 16), (_means, ("start", "count"), 4),
    (_topk, ("q", "m"), 16), (_topk, ("sl", "idx", "ns"), 4),
    (_project, ("h", "w", "q", "ki", "k8", "v8"), 16), (_project, ("start", "count", "ks", "vs"), 4)])
def test_pointers(call, names, align):
    sh = _shape()
    for n in names:
        assert call(sh, **{n: None}) == -1, n
        assert call(sh, **{n: ctypes.c_void_p(0x10008 if align == 16 else 0x10002)}) == -1, n
    if call in (_sparse, _dense):
        assert call(sh, lse=MIS) == -1
    if call in (_dense, _topk):
        assert call(_shape(causal=True), qp=None) == -1


def test_workspaces():
    sh = _shape(batch=1, max_len=8192, top_k=2048)
    for call, op, arg in ((_sparse, B.CLSA_OP_ATTN8, 0), (_dense, B.CLSA_OP_DENSE8, 0),
                          (_topk, B.CLSA_OP_BLOCK_TOPK, 64), (_project, B.CLSA_OP_PROJECT8, 0)):
        need = B.clsa_workspace_bytes(sh, op, arg)
        assert need > 0 and need % 256 == 0
        assert call(sh, ws=None, wsb=need) == -3
        assert call(sh, ws=A, wsb=need - 1) == -3
        assert call(sh, ws=ctypes.c_void_p(0x10010), wsb=need) == -3
    assert B.clsa_workspace_bytes(sh, B.CLSA_OP_BLOCK_TOPK, 0) == 0   # the block is asked for
    assert B.clsa_workspace_bytes(sh, B.CLSA_OP_BLOCK_TOPK, 24) == 0
    assert B.clsa_workspace_bytes(_shape(head_dim=64), B.CLSA_OP_ATTN8) == 0
    assert _project(sh, d=0) == -1 and _project(sh, d=500) == -2 and _project(sh, d=8704) == -2
    # a list of whole blocks
    assert _topk(_shape(top_k=100), ws=A, wsb=1 << 30) == -1
    assert _topk(_shape(top_k=32), ws=A, wsb=1 << 30) == -1
    assert B.clsa_workspace_bytes(_shape(top_k=100), B.CLSA_OP_BLOCK_TOPK, 64) == 0


def test_reference_rounding_is_the_formats():
    """The tests' e4m3 encoder against torch's conversion, over every bf16 value within 448."""
    bits = np.arange(65536, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    x = x[np.abs(x) <= 448]
    t = torch.from_numpy(x.copy()).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(C.encode(x.astype(np.float64)), t)
    assert np.array_equal(C.VALUES[np.arange(127)], torch.arange(127, dtype=torch.uint8)
                          .view(torch.float8_e4m3fn).double().numpy())


def test_binding_refuses_what_is_no_gpu_tensor():
    t = torch.zeros(16)
    with pytest.raises(ValueError, match="k must be a GPU tensor"):
        B.clsa_cache_append8(_shape(), 64, t, t, t, t, None, t, t, t, t)
    with pytest.raises(ValueError, match="ws must be a GPU tensor"):
        B.clsa_sparse_attn8(_shape(), 64, *[None] * 10, t)
    with pytest.raises(TypeError, match="q_idx must be a torch.Tensor"):
        B.clsa_block_topk(_shape(), 64, [1.0], t, None, t, None, t, t)
    with pytest.raises(B.ClsaError, match="CLSA_ERR_INVALID_ARG"):
        B.clsa_block_means(_shape(), 64, None, None, None, None, None, stream=types.SimpleNamespace(cuda_stream=0))


def test_binding_where_torch_has_no_raw_stream_handle(monkeypatch):
    """Such a torch loads the binding; a call takes the handle of torch's stream object."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    spec = importlib.util.spec_from_file_location("binding_alone", B.__file__)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    asked = []
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda device=None: asked.append(device) or types.SimpleNamespace(cuda_stream=0))
    with pytest.raises(m.ClsaError, match="CLSA_ERR_INVALID_ARG"):
        m.clsa_block_means(m.make_shape(2, 1, 1024, 128), 64, None, None, None, None, None)
    assert asked == [0]
