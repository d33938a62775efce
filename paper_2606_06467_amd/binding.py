"""Thin Python binding of libclsa (include/clsa.h): argument marshalling only.

Every function here has the name of the C entry point it wraps and takes
torch tensors that already live on the GPU; it passes their device pointers,
the shape struct and a HIP stream to the library, and raises ``ClsaError`` when
the library returns an error status.  No step of the path runs in Python, and
there is no fallback: if ``libclsa.so`` is missing the first call raises.
"""
from __future__ import annotations

import array
import ctypes
import math
import os
from typing import Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libclsa.so")

CLSA_OK = 0
CLSA_ERR_INVALID_ARG = -1
CLSA_ERR_UNSUPPORTED = -2
CLSA_ERR_WORKSPACE = -3
CLSA_ERR_HIP = -4
CLSA_ERR_SCRATCH_LIMIT = -5
CLSA_NOALLOC_SCRATCH_BYTES = 32 << 20

CLSA_OP_INDEX = 0
CLSA_OP_TOPK = 1
CLSA_OP_ATTN = 2
CLSA_OP_DECODE = 3
CLSA_OP_DENSE = 4
CLSA_OP_KD_TARGET = 5
CLSA_OP_KD_LOSS = 6
CLSA_OP_ATTN8 = 7
CLSA_OP_DENSE8 = 8
CLSA_OP_BLOCK_TOPK = 9
CLSA_OP_PROJECT8 = 10
CLSA_OP_ADAPTED = 11
CLSA_OP_ADAPTED8 = 12
CLSA_OP_NORM_GRAD = 13
CLSA_OP_PAGES_RESERVE = 14
CLSA_OP_PAGES_COMPACT = 15


class ClsaError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {clsa_status_string(status)} ({status})")
        self.status = status


class ClsaShape(ctypes.Structure):
    """Mirror of ``clsa_shape``."""
    _fields_ = [("batch", ctypes.c_int32), ("n_q", ctypes.c_int32),
                ("idx_heads", ctypes.c_int32), ("idx_dim", ctypes.c_int32),
                ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float)]


class ClsaPaged(ctypes.Structure):
    """Mirror of ``clsa_paged``."""
    _fields_ = [("data", ctypes.c_void_p), ("page_bytes", ctypes.c_int64)]


def make_shape(batch: int, n_q: int, max_len: int, top_k: int, *, idx_heads: int = 4,
               idx_dim: int = 64, q_heads: int = 32, kv_heads: int = 8, head_dim: int = 128,
               page_size: int = 0, max_pages: int = 0, causal: bool = False,
               softmax_scale: Optional[float] = None) -> ClsaShape:
    if softmax_scale is None:
        softmax_scale = 1.0 / math.sqrt(head_dim)
    return ClsaShape(batch, n_q, idx_heads, idx_dim, q_heads, kv_heads, head_dim, max_len,
                     page_size, max_pages, top_k, int(bool(causal)), softmax_scale)


_lib_handle = None


def lib() -> ctypes.CDLL:
    """The loaded libclsa.so (raises if it has not been built)."""
    global _lib_handle
    if _lib_handle is not None:
        return _lib_handle
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "(there is no fallback implementation)")
    L = ctypes.CDLL(LIB_PATH)
    P, SP = ctypes.c_void_p, ctypes.POINTER(ClsaShape)
    i32, i64, sz, dbl = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_double
    sig = {
        "clsa_workspace_bytes": (sz, [SP, i32, i32]),
        "clsa_index_scores": (i32, [SP, P, P, P, P, P, P, P]),
        "clsa_topk": (i32, [SP, P, P, P, P, P, P, sz, P]),
        "clsa_sparse_attn": (i32, [SP, P, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_decode_step": (i32, [SP, P, P, P, P, P, P, P, i32, P, P, P, P, P, P, sz, P]),
        "clsa_decode_step_noalloc": (i32, [SP, P, P, P, P, P, P, P, i32, P, P, P, P, P, P]),
        "clsa_decode_step_grouped": (i32, [SP, P, i64, P, i64, P, P, P, P, P, i32, i32, P, P, P,
                                           P, P, P, sz, P]),
        "clsa_dense_attn": (i32, [SP, P, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_project_append": (i32, [SP, i32, P, P, P, P, P, P, P, P, P]),
        "clsa_kd_target": (i32, [SP, i32, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_kd_loss": (i32, [SP, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_cache_append8": (i32, [SP, i32, P, P, P, P, P, P, P, P, P, P]),
        "clsa_project_append8": (i32, [SP, i32, i32, P, P, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_sparse_attn8": (i32, [SP, i32, P, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_dense_attn8": (i32, [SP, i32, P, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_block_means": (i32, [SP, i32, P, P, P, P, P, P]),
        "clsa_block_topk": (i32, [SP, i32, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_project_append_adapted": (i32, [SP, i32, i32, i32, P, P, P, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_project_append8_adapted": (i32, [SP, i32, i32, i32, i32, P, P, P, P, P, P, P, P, P, P, P, P, P,
                                               P, P, P, sz, P]),
        "clsa_residual_norm": (i32, [SP, i32, dbl, i32, P, P, P, P, P, P, P, P, P]),
        "clsa_residual_norm_grad": (i32, [SP, i32, P, P, P, P, P, P, P, P, sz, P]),
        "clsa_pages_fork": (i32, [SP, i32, P, P, P, P, P]),
        "clsa_pages_reserve": (i32, [SP, i32, i32, P, P, P, P, P, P, P, sz, P]),
        "clsa_pages_compact": (i32, [SP, i32, i32, P, P, P, P, P, sz, P]),
        "clsa_pages_copy": (i32, [i32, i32, P, i32, P, P, P]),
        "clsa_status_string": (ctypes.c_char_p, [i32]),
        "clsa_set_phase_events": (i32, [ctypes.POINTER(P), i32]),
        "clsa_get_device_error": (i32, [ctypes.POINTER(ctypes.c_uint32)]),
    }
    for name, (res, args) in sig.items():
        f = getattr(L, name)
        f.restype, f.argtypes = res, args
    _lib_handle = L
    return L


def _ptr(t: Optional[torch.Tensor], name: str):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _check(status: int, where: str) -> None:
    if status != CLSA_OK:
        raise ClsaError(status, where)


def clsa_status_string(status: int) -> str:
    return lib().clsa_status_string(int(status)).decode()


def clsa_workspace_bytes(shape: ClsaShape, op: int, n_layers: int = 0) -> int:
    return int(lib().clsa_workspace_bytes(ctypes.byref(shape), int(op), int(n_layers)))


def clsa_index_scores(shape, q_idx, k_idx, page_table, seq_lens, q_pos, scores, stream=None):
    _check(lib().clsa_index_scores(ctypes.byref(shape), _ptr(q_idx, "q_idx"), _ptr(k_idx, "k_idx"),
                                   _ptr(page_table, "page_table"), _ptr(seq_lens, "seq_lens"),
                                   _ptr(q_pos, "q_pos"), _ptr(scores, "scores"), _stream(stream)),
           "clsa_index_scores")


def clsa_topk(shape, scores, seq_lens, q_pos, idx, n_sel, ws=None, stream=None):
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().clsa_topk(ctypes.byref(shape), _ptr(scores, "scores"), _ptr(seq_lens, "seq_lens"),
                           _ptr(q_pos, "q_pos"), _ptr(idx, "idx"), _ptr(n_sel, "n_sel"),
                           _ptr(ws, "ws"), wsb, _stream(stream)), "clsa_topk")


def clsa_sparse_attn(shape, q, k_cache, v_cache, page_table, idx, n_sel, out, lse=None, ws=None,
                     stream=None):
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().clsa_sparse_attn(ctypes.byref(shape), _ptr(q, "q"), _ptr(k_cache, "k_cache"),
                                  _ptr(v_cache, "v_cache"), _ptr(page_table, "page_table"),
                                  _ptr(idx, "idx"), _ptr(n_sel, "n_sel"), _ptr(out, "out"),
                                  _ptr(lse, "lse"), _ptr(ws, "ws"), wsb, _stream(stream)),
           "clsa_sparse_attn")


def clsa_decode_step(shape, q_idx, k_idx, k_cache, v_cache, page_table, seq_lens, q_pos,
                     q_layers, out_layers, lse_layers, idx, n_sel, ws, stream=None):
    n_layers = 0 if q_layers is None else int(q_layers.shape[0])
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().clsa_decode_step(ctypes.byref(shape), _ptr(q_idx, "q_idx"), _ptr(k_idx, "k_idx"),
                                  _ptr(k_cache, "k_cache"), _ptr(v_cache, "v_cache"),
                                  _ptr(page_table, "page_table"), _ptr(seq_lens, "seq_lens"),
                                  _ptr(q_pos, "q_pos"), n_layers, _ptr(q_layers, "q_layers"),
                                  _ptr(out_layers, "out_layers"), _ptr(lse_layers, "lse_layers"),
                                  _ptr(idx, "idx"), _ptr(n_sel, "n_sel"), _ptr(ws, "ws"), wsb,
                                  _stream(stream)), "clsa_decode_step")


def clsa_decode_step_noalloc(shape, q_idx, k_idx, k_cache, v_cache, page_table, seq_lens, q_pos,
                             q_layers, out_layers, lse_layers, idx, n_sel, stream=None):
    """clsa_decode_step on the library's fixed per-device scratch (no workspace)."""
    n_layers = 0 if q_layers is None else int(q_layers.shape[0])
    _check(lib().clsa_decode_step_noalloc(
        ctypes.byref(shape), _ptr(q_idx, "q_idx"), _ptr(k_idx, "k_idx"), _ptr(k_cache, "k_cache"),
        _ptr(v_cache, "v_cache"), _ptr(page_table, "page_table"), _ptr(seq_lens, "seq_lens"),
        _ptr(q_pos, "q_pos"), n_layers, _ptr(q_layers, "q_layers"), _ptr(out_layers, "out_layers"),
        _ptr(lse_layers, "lse_layers"), _ptr(idx, "idx"), _ptr(n_sel, "n_sel"), _stream(stream)),
        "clsa_decode_step_noalloc")


def clsa_decode_step_grouped(shape, q_idx, q_idx_group_stride, k_idx, k_idx_group_stride,
                             k_cache, v_cache, page_table, seq_lens, q_pos, group, q_layers,
                             out_layers, lse_layers, idx, n_sel, ws, stream=None):
    """Strides in bf16 elements between the index queries / keys of consecutive sets."""
    n_layers = 0 if q_layers is None else int(q_layers.shape[0])
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().clsa_decode_step_grouped(
        ctypes.byref(shape), _ptr(q_idx, "q_idx"), int(q_idx_group_stride), _ptr(k_idx, "k_idx"),
        int(k_idx_group_stride), _ptr(k_cache, "k_cache"), _ptr(v_cache, "v_cache"),
        _ptr(page_table, "page_table"), _ptr(seq_lens, "seq_lens"), _ptr(q_pos, "q_pos"),
        n_layers, int(group), _ptr(q_layers, "q_layers"), _ptr(out_layers, "out_layers"),
        _ptr(lse_layers, "lse_layers"), _ptr(idx, "idx"), _ptr(n_sel, "n_sel"), _ptr(ws, "ws"),
        wsb, _stream(stream)), "clsa_decode_step_grouped")


def clsa_dense_attn(shape, q, k_cache, v_cache, page_table, seq_lens, q_pos, out, lse=None,
                    ws=None, stream=None):
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().clsa_dense_attn(ctypes.byref(shape), _ptr(q, "q"), _ptr(k_cache, "k_cache"),
                                 _ptr(v_cache, "v_cache"), _ptr(page_table, "page_table"),
                                 _ptr(seq_lens, "seq_lens"), _ptr(q_pos, "q_pos"),
                                 _ptr(out, "out"), _ptr(lse, "lse"), _ptr(ws, "ws"), wsb,
                                 _stream(stream)), "clsa_dense_attn")


def clsa_project_append(shape, d_model, h, w, pos, page_table, q_idx, k_idx, k_cache, v_cache,
                        stream=None):
    _check(lib().clsa_project_append(ctypes.byref(shape), int(d_model), _ptr(h, "h"), _ptr(w, "w"),
                                     _ptr(pos, "pos"), _ptr(page_table, "page_table"),
                                     _ptr(q_idx, "q_idx"), _ptr(k_idx, "k_idx"),
                                     _ptr(k_cache, "k_cache"), _ptr(v_cache, "v_cache"),
                                     _stream(stream)), "clsa_project_append")


def clsa_kd_target(shape, n_layers, q_layers, k_cache, page_table, seq_lens, q_pos, abar,
                   ws=None, stream=None, lse_layers=None):
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().clsa_kd_target(ctypes.byref(shape), int(n_layers), _ptr(q_layers, "q_layers"),
                                _ptr(k_cache, "k_cache"), _ptr(page_table, "page_table"),
                                _ptr(seq_lens, "seq_lens"), _ptr(q_pos, "q_pos"),
                                _ptr(lse_layers, "lse_layers"), _ptr(abar, "abar"),
                                _ptr(ws, "ws"), wsb, _stream(stream)), "clsa_kd_target")


def clsa_kd_loss(shape, abar, q_idx, k_idx, page_table, seq_lens, q_pos, loss, dq_idx, dk_idx,
                 ws=None, stream=None):
    wsb = 0 if ws is None else ws.numel() * ws.element_size()
    _check(lib().clsa_kd_loss(ctypes.byref(shape), _ptr(abar, "abar"), _ptr(q_idx, "q_idx"),
                              _ptr(k_idx, "k_idx"), _ptr(page_table, "page_table"),
                              _ptr(seq_lens, "seq_lens"), _ptr(q_pos, "q_pos"),
                              _ptr(loss, "loss"), _ptr(dq_idx, "dq_idx"), _ptr(dk_idx, "dk_idx"),
                              _ptr(ws, "ws"), wsb, _stream(stream)), "clsa_kd_loss")


_Tensor = torch.Tensor


def _stream_object(device):
    return torch.cuda.current_stream(device).cuda_stream


# The current stream's raw handle: making a torch Stream object takes 3 us, as long as the
# library's call.  It is no public name of torch, and a torch built without a GPU lacks it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _stream_object)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


# As functions: a call of a method is a third slower, and these three are most of a call's time here.
_get_device, _is_contiguous, _data_ptr = _Tensor.get_device, _Tensor.is_contiguous, _Tensor.data_ptr


def _call(where, shape, block, names, tensors, ws, stream, sizes=(), device=-1):
    """An entry point of the 8-bit cache or of what came after it: numbers after the block (or
    d_model, or the pool's pages), its tensors and their names, and its workspace (False: it takes
    none).  The call runs on the tensors' device (that of tensors among the numbers: device); their
    stream is the current one of that device unless one is given."""
    args, given = [*sizes], device
    append = args.append
    try:
        for t in tensors:
            if t is None:
                append(None)
            elif _get_device(t) == device >= 0 and _is_contiguous(t):
                append(_data_ptr(t))
            else:
                at = _get_device(t)
                if device >= 0 or at < 0 or not _is_contiguous(t):
                    _refuse(names[len(args) - len(sizes)], t)
                device = at
                append(_data_ptr(t))
    except TypeError:  # no tensor
        _refuse(names[len(args) - len(sizes)], t)
    if isinstance(ws, _Tensor):
        if ws.get_device() != device or device < 0 or not ws.is_contiguous():
            _refuse("ws", ws)
        args += ws.data_ptr(), ws.nbytes
    elif ws is None:
        args += None, 0
    if device >= 0 and device != _current_device():
        with torch.cuda.device(device):
            return _call(where, shape, block, names, tensors, ws, stream, sizes, given)
    raw = _raw_stream(max(device, 0)) if stream is None else stream.cuda_stream
    head = (block,) if shape is None else (ctypes.byref(shape), block)
    status = getattr(_lib_handle or lib(), where)(*head, *args, raw)
    if status != CLSA_OK:
        raise ClsaError(status, where)


def _refuse(name, t):
    _ptr(t, name)  # what is wrong with it alone
    raise ValueError(f"{name} is on another device than the arguments before it")


def clsa_cache_append8(shape, block, k, v, start, count, page_table, k8, v8, k_scale, v_scale,
                       stream=None):
    _call("clsa_cache_append8", shape, block,
          ("k", "v", "start", "count", "page_table", "k8", "v8", "k_scale", "v_scale"),
          (k, v, start, count, page_table, k8, v8, k_scale, v_scale), False, stream)


def clsa_project_append8(shape, block, d_model, h, w, start, count, page_table, q_idx, k_idx, k8, v8,
                         k_scale, v_scale, ws=None, stream=None):
    _call("clsa_project_append8", shape, block,
          ("h", "w", "start", "count", "page_table", "q_idx", "k_idx", "k8", "v8", "k_scale", "v_scale"),
          (h, w, start, count, page_table, q_idx, k_idx, k8, v8, k_scale, v_scale), ws, stream,
          (d_model,))


def clsa_sparse_attn8(shape, block, q, k8, v8, k_scale, v_scale, page_table, idx, n_sel, out,
                      lse=None, ws=None, stream=None):
    _call("clsa_sparse_attn8", shape, block,
          ("q", "k8", "v8", "k_scale", "v_scale", "page_table", "idx", "n_sel", "out", "lse"),
          (q, k8, v8, k_scale, v_scale, page_table, idx, n_sel, out, lse), ws, stream)


def clsa_dense_attn8(shape, block, q, k8, v8, k_scale, v_scale, page_table, seq_lens, q_pos, out,
                     lse=None, ws=None, stream=None):
    _call("clsa_dense_attn8", shape, block,
          ("q", "k8", "v8", "k_scale", "v_scale", "page_table", "seq_lens", "q_pos", "out", "lse"),
          (q, k8, v8, k_scale, v_scale, page_table, seq_lens, q_pos, out, lse), ws, stream)


def clsa_block_means(shape, block, k_idx, start, count, page_table, means, stream=None):
    _call("clsa_block_means", shape, block, ("k_idx", "start", "count", "page_table", "means"),
          (k_idx, start, count, page_table, means), False, stream)


def clsa_block_topk(shape, block, q_idx, means, page_table, seq_lens, q_pos, idx, n_sel, ws=None,
                    stream=None):
    _call("clsa_block_topk", shape, block,
          ("q_idx", "means", "page_table", "seq_lens", "q_pos", "idx", "n_sel"),
          (q_idx, means, page_table, seq_lens, q_pos, idx, n_sel), ws, stream)


def _adapter_sizes(shape, d_model, a, b, alpha, adapter):
    """Number and rank of the adapters a [adapters, rank, d_model], b [adapters, features, rank], whose
    other sizes, and those of alpha and adapter, the library takes from the shape."""
    for name, t in (("a", a), ("b", b)):
        if not isinstance(t, _Tensor) or t.dim() != 3:
            raise ValueError(f"{name} must be a tensor of three dimensions")
    n, rank, width = a.shape
    held, features, held_rank = b.shape
    if held != n or held_rank != rank:
        raise ValueError("a and b must hold the same adapters, of one rank")
    if width != d_model:
        raise ValueError(f"a must hold vectors of d_model {d_model} values, not {width}")
    if features != 512 + 2 * shape.kv_heads * shape.head_dim:
        raise ValueError(f"b must hold the shape's {512 + 2 * shape.kv_heads * shape.head_dim} features, not {features}")
    if isinstance(alpha, _Tensor) and alpha.numel() < n:
        raise ValueError(f"alpha must hold a factor for each of the {n} adapters")
    if isinstance(adapter, _Tensor) and adapter.numel() < shape.batch:
        raise ValueError(f"adapter must hold a number for each of the {shape.batch} sequences")
    return n, rank


def clsa_project_append_adapted(shape, d_model, h, w, a, b, alpha, adapter, pos, page_table, q_idx, k_idx,
                                k_cache, v_cache, ws=None, stream=None):
    """a: [adapters, rank, d_model], b: [adapters, features, rank]."""
    _call("clsa_project_append_adapted", shape, d_model,
          ("h", "w", "a", "b", "alpha", "adapter", "pos", "page_table", "q_idx", "k_idx", "k_cache", "v_cache"),
          (h, w, a, b, alpha, adapter, pos, page_table, q_idx, k_idx, k_cache, v_cache), ws, stream,
          _adapter_sizes(shape, d_model, a, b, alpha, adapter))


def clsa_project_append8_adapted(shape, block, d_model, h, w, a, b, alpha, adapter, start, count, page_table,
                                 q_idx, k_idx, k8, v8, k_scale, v_scale, ws=None, stream=None):
    _call("clsa_project_append8_adapted", shape, block,
          ("h", "w", "a", "b", "alpha", "adapter", "start", "count", "page_table", "q_idx", "k_idx", "k8", "v8",
           "k_scale", "v_scale"),
          (h, w, a, b, alpha, adapter, start, count, page_table, q_idx, k_idx, k8, v8, k_scale, v_scale), ws,
          stream, (d_model, *_adapter_sizes(shape, d_model, a, b, alpha, adapter)))


def clsa_residual_norm(shape, d_model, eps, x, residual, weight, sum=None, y=None, y8=None, y_scale=None,
                       rstd=None, stream=None, *, group=128):
    _call("clsa_residual_norm", shape, d_model,
          ("x", "residual", "weight", "sum", "y", "y8", "y_scale", "rstd"),
          (x, residual, weight, sum, y, y8, y_scale, rstd), False, stream, (eps, group))


def clsa_residual_norm_grad(shape, d_model, s, rstd, weight, dy, dsum, dx, dweight, ws=None, stream=None):
    _call("clsa_residual_norm_grad", shape, d_model,
          ("s", "rstd", "weight", "dy", "dsum", "dx", "dweight"),
          (s, rstd, weight, dy, dsum, dx, dweight), ws, stream)


def _paged(tensors, pages):
    """The host array of a paged cache's tensors (held by the caller while it is in use), its length
    and address as arguments, and the tensors' device."""
    fields, device = array.array("q"), -1  # data and page_bytes of each
    for i, t in enumerate(tensors):
        if not isinstance(t, _Tensor):
            raise TypeError(f"tensors[{i}] must be a torch.Tensor")
        at = _get_device(t)
        if at < 0 or not _is_contiguous(t) or (at != device and device >= 0):
            _refuse(f"tensors[{i}]", t)
        if t.dim() < 1 or t.size(0) != pages:
            raise ValueError(f"tensors[{i}] must have one row for each of the {pages} pages of refs")
        device = at
        fields.append(_data_ptr(t))
        fields.append(t.nbytes // pages)
    return fields, (len(tensors), fields.buffer_info()[0]), device


def clsa_pages_fork(shape, parent, page_table, seq_lens, refs, stream=None):
    _call("clsa_pages_fork", shape, refs.numel(), ("parent", "page_table", "seq_lens", "refs"),
          (parent, page_table, seq_lens, refs), False, stream)


def clsa_pages_reserve(shape, tensors, start, count, page_table, refs, missing, ws=None, stream=None):
    """tensors: the cache's tensors, each with a leading dimension of refs.numel() pages."""
    pages = refs.numel()
    held, sizes, device = _paged(tensors, pages)
    _call("clsa_pages_reserve", shape, pages, ("start", "count", "page_table", "refs", "missing"),
          (start, count, page_table, refs, missing), ws, stream, sizes, device)


def clsa_pages_compact(shape, tensors, page_table, refs, bound, ws=None, stream=None):
    pages = refs.numel()
    held, sizes, device = _paged(tensors, pages)
    _call("clsa_pages_compact", shape, pages, ("page_table", "refs", "bound"), (page_table, refs, bound), ws,
          stream, sizes, device)


def clsa_pages_copy(tensors, src, dst, stream=None):
    """Pages src[i] to dst[i] of every tensor (they have the same number of pages)."""
    pages = tensors[0].shape[0] if tensors else 1
    held, sizes, device = _paged(tensors, pages)
    if src.numel() != dst.numel():
        raise ValueError("src and dst must have one length")
    _call("clsa_pages_copy", None, pages, ("src", "dst"), (src, dst), False, stream, (*sizes, src.numel()),
          device)


CLSA_DEVERR_SEQ_LEN = 1
CLSA_DEVERR_N_SEL = 2
CLSA_DEVERR_APPEND = 4
CLSA_DEVERR_ADAPTER = 8
CLSA_DEVERR_PAGES = 16


def clsa_get_device_error() -> int:
    """Device error bits (CLSA_DEVERR_*) raised since the last call on the
    current device, cleared by the call.  Synchronises the device."""
    v = ctypes.c_uint32(0)
    _check(lib().clsa_get_device_error(ctypes.byref(v)), "clsa_get_device_error")
    return int(v.value)


def clsa_set_phase_events(events: Optional[Sequence[int]]) -> None:
    """events: 4 + 2m raw hipEvent_t handles (ints): the four phase marks, then a
    (before, after) pair around the attention kernel of each of the first m
    layers; None switches the hook off."""
    if not events:
        _check(lib().clsa_set_phase_events(None, 0), "clsa_set_phase_events")
        return
    arr = (ctypes.c_void_p * len(events))(*[ctypes.c_void_p(int(e)) for e in events])
    _check(lib().clsa_set_phase_events(arr, len(events)), "clsa_set_phase_events")


def workspace(shape: ClsaShape, op: int, n_layers: int = 0, device="cuda") -> Optional[torch.Tensor]:
    """A device byte tensor large enough for ``op`` (None if none is needed); for
    CLSA_OP_BLOCK_TOPK ``n_layers`` is the tokens per block, for CLSA_OP_ADAPTED and
    CLSA_OP_ADAPTED8 the rank, for CLSA_OP_NORM_GRAD d_model, for CLSA_OP_PAGES_COMPACT the
    pool's pages."""
    n = clsa_workspace_bytes(shape, op, n_layers)
    if n == 0:
        return None
    return torch.empty(n, dtype=torch.uint8, device=device)


HIP_EVENT_DISABLE_SYSTEM_FENCE = 0x20000000  # hipEventDisableSystemFence


class HipEvents:
    """Raw HIP events (libamdhip64) for timing work on a given stream.

    ``timing_only`` events skip the system-scope fence that an event record
    otherwise performs (a cache write-back and invalidate, which both costs time
    and slows the work after it); read them only after the device has been
    synchronised."""

    def __init__(self, n: int, timing_only: bool = False):
        self._hip = ctypes.CDLL("libamdhip64.so")
        self._hip.hipEventCreateWithFlags.argtypes = [ctypes.POINTER(ctypes.c_void_p),
                                                      ctypes.c_uint]
        self._hip.hipEventRecord.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        self._hip.hipEventSynchronize.argtypes = [ctypes.c_void_p]
        self._hip.hipEventElapsedTime.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_void_p,
                                                  ctypes.c_void_p]
        self._hip.hipEventDestroy.argtypes = [ctypes.c_void_p]
        self.handles = []
        for _ in range(n):
            h = ctypes.c_void_p()
            flags = HIP_EVENT_DISABLE_SYSTEM_FENCE if timing_only else 0
            if self._hip.hipEventCreateWithFlags(ctypes.byref(h), flags) != 0:
                raise RuntimeError("hipEventCreateWithFlags failed")
            self.handles.append(h.value)

    def record(self, i: int, stream=None) -> None:
        if self._hip.hipEventRecord(ctypes.c_void_p(self.handles[i]), _stream(stream)) != 0:
            raise RuntimeError("hipEventRecord failed")

    def elapsed_ms(self, i: int, j: int) -> float:
        self._hip.hipEventSynchronize(ctypes.c_void_p(self.handles[j]))
        ms = ctypes.c_float()
        if self._hip.hipEventElapsedTime(ctypes.byref(ms), ctypes.c_void_p(self.handles[i]),
                                         ctypes.c_void_p(self.handles[j])) != 0:
            raise RuntimeError("hipEventElapsedTime failed")
        return float(ms.value)

    def close(self) -> None:
        for h in self.handles:
            self._hip.hipEventDestroy(ctypes.c_void_p(h))
        self.handles = []


def bf16_from_bits(bits, device="cuda") -> torch.Tensor:
    """A bfloat16 device tensor holding the given uint16 bit patterns (numpy array)."""
    import numpy as np
    arr = np.ascontiguousarray(bits, dtype=np.uint16)
    return torch.from_numpy(arr.view(np.int16)).view(torch.bfloat16).to(device)


def bits_from_bf16(t: torch.Tensor):
    """uint16 numpy bit patterns of a bfloat16 tensor."""
    import numpy as np
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
