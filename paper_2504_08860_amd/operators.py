"""Binding of the operators beside the sparse products (``include/hbp.h``): 4-bit matrices, residual norms, token log probabilities.

Argument marshalling only, as in the package itself, whose names these functions are reached by.  Tensors are checked for device,
type and shape; rows may lie further apart than they are long (the last dimension is contiguous).  A call runs on torch's current
stream, or on the ``stream`` that is given; what it needs in the meantime is a ``workspace`` tensor, which is allocated by the call, on
that stream, unless one is given.  Outputs are written in place; which inputs they may share memory with is said in the header.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools

import paper_2504_08860_amd as _core

GATE_NONE, GATE_CHANNEL, GATE_TOKEN, GATE_FULL = 0, 1, 2, 3


class hbp_q4_matrix_t(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("zeros", ctypes.c_void_p), ("n_rows", ctypes.c_int64),
                ("n_cols", ctypes.c_int64), ("group", ctypes.c_int32), ("scale_type", ctypes.c_int32)]


class hbp_norms_t(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("width", ctypes.c_int64), ("type", ctypes.c_int32), ("gate_kind", ctypes.c_int32),
                ("w_post", ctypes.c_void_p), ("w_pre", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("ldg", ctypes.c_int64),
                ("scale", ctypes.c_float), ("eps", ctypes.c_float)]


_torch = _uint8 = _i32 = _i64 = _f32 = None
_types = {}  # the library's numbers of torch's value types; set, as those above, with the library's argument types


def declare(L) -> None:
    """Sets the argument types of the operators' entry points."""
    global _torch, _uint8, _i32, _i64, _f32
    import torch
    _torch, _uint8, _i32, _i64, _f32 = torch, torch.uint8, torch.int32, torch.int64, torch.float32
    _types.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
    vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    matrix, norms, size_out = ctypes.POINTER(hbp_q4_matrix_t), ctypes.POINTER(hbp_norms_t), ctypes.POINTER(size)
    L.hbp_q4_pack.argtypes = L.hbp_q4_unpack.argtypes = [matrix, i32, vp, i64, vp]
    L.hbp_q4_mv.argtypes = [matrix, i32, vp, i64, vp, i64, i64, vp]
    L.hbp_q4_mv_t.argtypes = [matrix, i32, vp, i64, vp, i64, i64, vp, size, vp]
    L.hbp_q4_mv_t_workspace.argtypes = [matrix, i64, size_out]
    L.hbp_residual_norms.argtypes = [norms] + [vp, i64] * 4 + [vp, vp]
    L.hbp_residual_norms_backward.argtypes = [norms] + [vp, i64] * 4 + [vp] + [vp, i64] * 2 + [vp, vp, vp, vp, size, vp]
    L.hbp_residual_norms_backward_workspace.argtypes = [norms, size_out]
    L.hbp_token_logprobs.argtypes = [i32, vp, i64, i64, i64, vp, i32, vp, vp, vp, i32, vp, vp, vp, size, vp]
    L.hbp_token_logprobs_workspace.argtypes = [i32, i64, i64, i32, size_out]
    L.hbp_token_logprobs_backward.argtypes = [i32, vp, i64, i64, i64, vp, i32] + [vp] * 5 + [i64, vp]


# (A small operator is 3 to 5 us of GPU time, and these checks are much of what a loop of them waits for.  A tensor's shape, strides, type,
# device and address cost 0.1 us each: each is asked for once, and the current device once a call.)
def _rows(t, what, shape, dtype, device):
    """(address, row stride) of a tensor of this shape and type on the device, rows contiguous in themselves."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == device:
        if len(shape) == 1:
            if t.is_contiguous():
                return t.data_ptr(), shape[0]
        else:
            apart, step = t.stride()
            if shape[0] < 2:
                apart = shape[1]
            if apart >= shape[1] and (step == 1 or shape[1] < 2):
                return t.data_ptr(), apart
    raise AssertionError(f"{what}: {dtype} tensor of shape {tuple(shape)} on the current CUDA device required, rows contiguous in themselves")


def _whole(t, what, shape, dtype, device):
    """Address of a contiguous tensor of this shape and type on the device; None for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    raise AssertionError(f"{what}: contiguous {dtype} tensor of shape {tuple(shape)} on the current CUDA device required")


def _on(stream):
    """Allocations of the block go to the stream that uses them: their memory may be handed out again, on that stream, as soon as the call is over."""
    if stream is None:
        return contextlib.nullcontext()
    return _torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else _torch.cuda.ExternalStream(int(stream)))


def _space(workspace, need, stream, device):
    """(address, bytes, what keeps it) of a workspace of at least ``need`` bytes."""
    if workspace is not None:
        assert workspace.get_device() == device and workspace.is_contiguous(), "workspace: contiguous tensor on the current CUDA device required"
        return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace
    if not need:
        return None, 0, None
    if stream is None:
        t = _torch.empty(need, dtype=_uint8, device="cuda")
    else:
        with _on(stream):
            t = _torch.empty(need, dtype=_uint8, device="cuda")
    return t.data_ptr(), need, t


# ------------------------------------------------------------------------------------ 4-bit matrices

def hbp_q4_shapes(n_rows: int, n_cols: int, group: int = 128):
    """Shapes of a 4-bit matrix's codes (uint8) and of its scales (and zero points)."""
    return (n_rows, (n_cols + 31) // 32 * 16), (n_rows, (n_cols + group - 1) // group)


def _matrix(codes, scales, zeros, n_cols, group, device):
    assert codes.dim() == 2, "codes: uint8 matrix required"
    n_rows = codes.shape[0]
    kind = scales.dtype
    assert kind in _types, "scales: float32, float16 or bfloat16 required"
    assert group > 0, "group: a number of columns required"
    groups = (n_rows, (n_cols + group - 1) // group)
    return hbp_q4_matrix_t(_whole(codes, "codes", (n_rows, (n_cols + 31) // 32 * 16), _uint8, device), _whole(scales, "scales", groups, kind, device),
                           _whole(zeros, "zeros", groups, kind, device), n_rows, n_cols, group, _types[kind])


def _start():
    """(the library, the current device)"""
    return _core._lib or _core.lib(), _core._current_device()


def hbp_q4_pack(w, codes, scales, group: int = 128, zeros=None, stream=None) -> None:
    """Rounds the matrix ``w`` [rows, cols] into ``codes``, ``scales`` and, if given, ``zeros`` (shapes: hbp_q4_shapes)."""
    L, device = _start()
    assert w.dtype in _types and w.dim() == 2, "w: matrix of float32, float16 or bfloat16 required"
    m = _matrix(codes, scales, zeros, w.shape[1], group, device)
    at, ld = _rows(w, "w", (m.n_rows, m.n_cols), w.dtype, device)
    _core._check(L.hbp_q4_pack(m, _types[w.dtype], at, ld, _core._stream_ptr(stream)), "hbp_q4_pack")


def hbp_q4_unpack(codes, scales, n_cols: int, group: int = 128, zeros=None, out=None, stream=None):
    """The values that the codes stand for [rows, n_cols]: in ``out``, or in a new float32 tensor."""
    L, device = _start()
    m = _matrix(codes, scales, zeros, n_cols, group, device)
    if out is None:
        with _on(stream):
            out = _torch.empty(codes.shape[0], n_cols, dtype=_torch.float32, device="cuda")
    assert out.dtype in _types, "out: float32, float16 or bfloat16 required"
    at, ld = _rows(out, "out", (m.n_rows, m.n_cols), out.dtype, device)
    _core._check(L.hbp_q4_unpack(m, _types[out.dtype], at, ld, _core._stream_ptr(stream)), "hbp_q4_unpack")
    return out


def _vectors(x, y, n_x, n_y, device):
    """(type, address and row stride of x and of y, how many vectors)"""
    dtype = x.dtype
    assert dtype in _types, "x: float32, float16 or bfloat16 required"
    one = x.dim() == 1
    count = 1 if one else x.shape[0]
    x_at, ldx = _rows(x, "x", (n_x,) if one else (count, n_x), dtype, device)
    y_at, ldy = _rows(y, "y", (n_y,) if one else (count, n_y), dtype, device)
    return _types[dtype], x_at, ldx, y_at, ldy, count


def hbp_q4_mv(codes, scales, x, y, group: int = 128, zeros=None, stream=None) -> None:
    """y = x W^T with the 4-bit matrix W [rows, cols]: ``x`` [cols] and ``y`` [rows], or [vectors, cols] and [vectors, rows]."""
    L, device = _start()
    assert x.dim(), "x: vector or matrix required"
    m = _matrix(codes, scales, zeros, x.shape[-1], group, device)
    status = L.hbp_q4_mv(m, *_vectors(x, y, m.n_cols, m.n_rows, device), _core._stream_ptr(stream))
    if status:
        raise _core.HbpError(status, "hbp_q4_mv")


@functools.lru_cache(maxsize=1024)
def _mv_t_bytes(n_rows, n_cols, group, scale_type, vectors):
    need = ctypes.c_size_t()
    m = hbp_q4_matrix_t(4096, 4096, None, n_rows, n_cols, group, scale_type)  # (sizes alone are looked at)
    _core._check(_core.lib().hbp_q4_mv_t_workspace(m, vectors, need), "hbp_q4_mv_t_workspace")
    return need.value


def hbp_q4_mv_t(codes, scales, x, y, group: int = 128, zeros=None, workspace=None, stream=None) -> None:
    """y = x W with the 4-bit matrix W [rows, cols], the gradient of hbp_q4_mv for its x: ``x`` [rows] and ``y`` [cols], or [vectors,
    rows] and [vectors, cols]."""
    L, device = _start()
    assert x.dim() and y.dim(), "x, y: vectors or matrices required"
    m = _matrix(codes, scales, zeros, y.shape[-1], group, device)
    v = _vectors(x, y, m.n_rows, m.n_cols, device)
    at, size, kept = _space(workspace, _mv_t_bytes(m.n_rows, m.n_cols, group, m.scale_type, v[5]), stream, device)
    status = L.hbp_q4_mv_t(m, *v, at, size, _core._stream_ptr(stream))
    if status:
        raise _core.HbpError(status, "hbp_q4_mv_t")


# ------------------------------------------------------------------------------------ residual norms

def _norms(shape, dtype, w_post, w_pre, gate, scale, eps, device):
    assert dtype in _types and len(shape) == 2, "h: matrix of float32, float16 or bfloat16 required"
    kind, at, ldg, wide = GATE_NONE, None, 0, (shape[1],)
    if gate is not None:
        dims = gate.dim()
        if dims == 1:
            kind, at = GATE_CHANNEL, _whole(gate, "gate", wide, dtype, device)
        elif dims == 2 and gate.shape[1] == 1 and shape[1] != 1:
            kind, at = GATE_TOKEN, _whole(gate, "gate", (shape[0], 1), dtype, device)
        else:
            kind = GATE_FULL
            at, ldg = _rows(gate, "gate", shape, dtype, device)
    return hbp_norms_t(shape[0], shape[1], _types[dtype], kind, _whole(w_post, "w_post", wide, dtype, device), _whole(w_pre, "w_pre", wide, dtype, device),
                       at, ldg, scale, eps)


def hbp_residual_norms(h, y, h_out, x_out, rstd=None, w_post=None, w_pre=None, gate=None, scale: float = 1.0, eps: float = 1e-6, stream=None) -> None:
    """h_out = h + scale gate norm(y) w_post, x_out = norm(h_out) w_pre, row by row of [tokens, width].  ``gate``: None, [width], [tokens, 1]
    or [tokens, width]; ``rstd`` float32 [tokens, 2]: both norms' factors, for the backward call."""
    L, device = _start()
    shape, dtype = h.shape, h.dtype
    n = _norms(shape, dtype, w_post, w_pre, gate, scale, eps, device)
    status = L.hbp_residual_norms(n, *_rows(h, "h", shape, dtype, device), *_rows(y, "y", shape, dtype, device), *_rows(h_out, "h_out", shape, dtype, device),
                                  *_rows(x_out, "x_out", shape, dtype, device), _whole(rstd, "rstd", (shape[0], 2), _f32, device),
                                  _core._stream_ptr(stream))
    if status:
        raise _core.HbpError(status, "hbp_residual_norms")


@functools.lru_cache(maxsize=1024)
def _norms_bytes(tokens, width, dtype_number):
    need = ctypes.c_size_t()
    n = hbp_norms_t(tokens, width, dtype_number, GATE_NONE, None, None, None, 0, 1.0, 1.0)  # (sizes alone are looked at)
    _core._check(_core.lib().hbp_residual_norms_backward_workspace(n, need), "hbp_residual_norms_backward_workspace")
    return need.value


def hbp_residual_norms_backward(d_h_out, d_x_out, h, y, rstd, d_h, d_y, d_w_post=None, d_w_pre=None, d_gate=None, w_post=None, w_pre=None,
                                gate=None, scale: float = 1.0, workspace=None, stream=None) -> None:
    """Gradients of hbp_residual_norms from those of its outputs (either may be None: zero), its inputs and ``rstd``.  ``d_w_post``, ``d_w_pre``
    and the ``d_gate`` of a [width] or [tokens, 1] gate are float32, that of a full gate has its type (and row stride)."""
    L, device = _start()
    shape, dtype = h.shape, h.dtype
    n = _norms(shape, dtype, w_post, w_pre, gate, scale, 1.0, device)
    wide, dg_at = (shape[1],), None
    if d_gate is not None:
        assert gate is not None, "d_gate: no gate was given"
        if n.gate_kind == GATE_FULL:
            dg_at, lddg = _rows(d_gate, "d_gate", shape, dtype, device)
            assert lddg == n.ldg, "d_gate: the gate's row stride required"
        else:
            dg_at = _whole(d_gate, "d_gate", gate.shape, _f32, device)
    none = (None, 0)
    at, size, kept = _space(workspace, _norms_bytes(n.tokens, n.width, n.type), stream, device)
    status = L.hbp_residual_norms_backward(
        n, *(none if d_h_out is None else _rows(d_h_out, "d_h_out", shape, dtype, device)),
        *(none if d_x_out is None else _rows(d_x_out, "d_x_out", shape, dtype, device)), *_rows(h, "h", shape, dtype, device),
        *_rows(y, "y", shape, dtype, device), _whole(rstd, "rstd", (shape[0], 2), _f32, device), *_rows(d_h, "d_h", shape, dtype, device),
        *_rows(d_y, "d_y", shape, dtype, device), _whole(d_w_post, "d_w_post", wide, _f32, device), _whole(d_w_pre, "d_w_pre", wide, _f32, device), dg_at,
        at, size, _core._stream_ptr(stream))
    if status:
        raise _core.HbpError(status, "hbp_residual_norms_backward")


# ------------------------------------------------------------------------------------ token log probabilities

def _ids(tokens, count, device):
    if tokens is None:
        return None, 0
    kind = tokens.dtype
    assert kind is _i64 or kind is _i32, "tokens: int32 or int64 required"
    return _whole(tokens, "tokens", (count,), kind, device), 8 if kind is _i64 else 4


@functools.lru_cache(maxsize=1024)
def _logprobs_bytes(dtype_number, tokens, vocabulary, top):
    need = ctypes.c_size_t()
    _core._check(_core.lib().hbp_token_logprobs_workspace(dtype_number, tokens, vocabulary, top, need), "hbp_token_logprobs_workspace")
    return need.value


def hbp_token_logprobs(logits, tokens, logp=None, entropy=None, lse=None, top_ids=None, top_logp=None, workspace=None, stream=None) -> None:
    """Of every row of ``logits`` [n, vocabulary]: the log probability of its token (``tokens`` [n], int32 or int64, negative: none), the entropy, the
    logarithm of the sum of exponentials (float32 [n] each) and the ``top_ids`` (int32) with their ``top_logp`` (float32), both [n, top]."""
    L, device = _start()
    shape, dtype = logits.shape, logits.dtype
    assert dtype in _types and len(shape) == 2, "logits: matrix of float32, float16 or bfloat16 required"
    count, vocabulary = shape
    assert (top_ids is None) == (top_logp is None), "top_ids and top_logp go together"
    top = 0
    if top_ids is not None:
        assert top_ids.dim() == 2, "top_ids: int32 matrix required"
        top = top_ids.shape[1]
    number, each, best = _types[dtype], (count,), (count, top)
    at, size, kept = _space(workspace, _logprobs_bytes(number, count, vocabulary, top), stream, device)
    z_at, ldz = _rows(logits, "logits", shape, dtype, device)
    status = L.hbp_token_logprobs(number, z_at, ldz, count, vocabulary, *_ids(tokens, count, device), _whole(logp, "logp", each, _f32, device),
                                  _whole(entropy, "entropy", each, _f32, device), _whole(lse, "lse", each, _f32, device), top,
                                  _whole(top_ids, "top_ids", best, _i32, device), _whole(top_logp, "top_logp", best, _f32, device), at, size,
                                  _core._stream_ptr(stream))
    if status:
        raise _core.HbpError(status, "hbp_token_logprobs")


def hbp_token_logprobs_backward(logits, tokens, lse, entropy, g_logp, g_entropy, d_logits, stream=None) -> None:
    """The gradient for ``logits``, of their type, from those of logp and entropy (float32 [n], either may be None: zero) and the forward call's
    ``lse`` and ``entropy``.  ``d_logits`` may be ``logits``."""
    L, device = _start()
    shape, dtype = logits.shape, logits.dtype
    assert dtype in _types and len(shape) == 2, "logits: matrix of float32, float16 or bfloat16 required"
    count, vocabulary = shape
    each = (count,)
    z_at, ldz = _rows(logits, "logits", shape, dtype, device)
    status = L.hbp_token_logprobs_backward(_types[dtype], z_at, ldz, count, vocabulary, *_ids(tokens, count, device), _whole(lse, "lse", each, _f32, device),
                                           _whole(entropy, "entropy", each, _f32, device), _whole(g_logp, "g_logp", each, _f32, device),
                                           _whole(g_entropy, "g_entropy", each, _f32, device), *_rows(d_logits, "d_logits", shape, dtype, device),
                                           _core._stream_ptr(stream))
    if status:
        raise _core.HbpError(status, "hbp_token_logprobs_backward")
