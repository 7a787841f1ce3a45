"""Binding of what a reader's training step does around its attention (include/plaid.h): embedding, dropout, layer norm, cross entropy
over a vocabulary, with their gradients.

Like `reader.py` this only marshals, and keeps nothing from one call for the next.  Autograd records none of the calls: each gradient
is a call of its own, and inputs that require a gradient are refused where it is enabled, those of the gradients' calls too (examples/reader.py
has the Functions).  Nor do they carry a forward-mode tangent on: inputs that have one are refused.
"""
from __future__ import annotations

import ctypes as ct
import struct
from typing import Optional, Tuple

import torch
from torch.autograd import forward_ad as _forward

from . import plaid as _p
from .reader import _DTYPES, _no_tangents, _workspace


class plaid_token_loss(ct.Structure):
    _fields_ = [("dtype", ct.c_int32), ("width", ct.c_int32), ("rows", ct.c_int64), ("vocabulary", ct.c_int64), ("scale", ct.c_float),
                ("hidden", ct.c_void_p), ("weight", ct.c_void_p), ("hidden_stride", ct.c_int64), ("weight_stride", ct.c_int64),
                ("targets", ct.c_void_p), ("loss", ct.c_void_p), ("lse", ct.c_void_p)]


def declare(lib: ct.CDLL) -> None:
    """Argument types of these functions."""
    P, i32, i64, f32, out64 = ct.c_void_p, ct.c_int32, ct.c_int64, ct.c_float, ct.POINTER(ct.c_int64)
    loss = ct.POINTER(plaid_token_loss)
    lib.plaid_embedding.argtypes = [P, i64, i64, i32, P, i64, f32, P, i32, ct.c_int, P]
    lib.plaid_embedding_backward.argtypes = [P, i64, i64, i32, P, i64, f32, i32, P, i32, P, i64, ct.c_int, P]
    lib.plaid_embedding_backward_workspace.argtypes = [i64, i64, i32, out64]
    lib.plaid_dropout.argtypes = [P, P, i64, f32, P, P, i32, ct.c_int, P]
    lib.plaid_layer_norm.argtypes = [P, i64, P, P, i64, i32, f32, P, P, i32, ct.c_int, P]
    lib.plaid_layer_norm_backward.argtypes = [P, i64, P, i64, P, P, i64, i32, P, P, P, i32, P, i64, ct.c_int, P]
    lib.plaid_layer_norm_backward_workspace.argtypes = [i64, i32, out64]
    lib.plaid_cross_entropy.argtypes = [loss, P, i64, ct.c_int, P]
    lib.plaid_cross_entropy_backward.argtypes = [loss, P, i64, P, P, P, i64, ct.c_int, P]
    lib.plaid_cross_entropy_workspace.argtypes = [loss, i32, out64]


def _states(t: torch.Tensor, name: str, dim: Optional[int] = 2) -> int:
    """Checks a tensor of states; its device's ordinal."""
    device = t.get_device() if isinstance(t, torch.Tensor) else -1
    if device < 0 or t.dtype not in _DTYPES or (dim is not None and t.dim() != dim):
        raise ValueError(f"{name} must be a CUDA tensor of dtype torch.bfloat16 or torch.float16" + ("" if dim is None else f" with {dim} dimensions"))
    return device


def _same(t: torch.Tensor, name: str, dtype: torch.dtype, shape, device: int) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.get_device() != device or t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be a tensor of dtype {dtype} and shape {tuple(shape)} on the device of the states")
    return t


def _not_recorded(backward: Optional[str], **tensors) -> None:
    """Called where autograd is enabled and one of the tensors may require a gradient; backward: the call that forms it, if there is one."""
    for name, t in tensors.items():
        if isinstance(t, torch.Tensor) and t.requires_grad:
            raise ValueError(f"{name} requires a gradient, which this call does not record: call it in torch.no_grad()" +
                             (f", or in a torch.autograd.Function whose backward calls {backward}" if backward else " (gradients of gradients are not formed)"))


_recording = torch.is_grad_enabled


def _rows(t: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """A matrix whose rows are contiguous, and from one row to the next."""
    if t.is_contiguous():
        return t, t.shape[1]
    row, one = t.stride()
    if one != 1 and t.shape[1] > 1:
        t = t.contiguous()
        return t, t.shape[1]
    return t, row if t.shape[0] > 1 else t.shape[1]


def _aligned_rows(t: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """The same where the kernels want rows of whole 16-byte pieces."""
    n, width = t.shape
    stride, one = t.stride()
    if n < 2:
        stride = width
    if (one != 1 and width > 1) or stride % 8 or stride >= 1 << 24 or t.data_ptr() % 16:
        if t.numel():
            t = t.clone(memory_format=torch.contiguous_format)
        stride = width
    return t, stride


def _parameter(t: Optional[torch.Tensor], name: str, x: torch.Tensor, width: int, device: int) -> Tuple[Optional[torch.Tensor], Optional[int]]:
    """A weight or bias of x's rows, and its address."""
    if t is None:
        return None, None
    if not isinstance(t, torch.Tensor) or t.get_device() != device or t.dtype is not x.dtype or t.dim() != 1 or t.shape[0] != width:
        raise ValueError(f"{name} must hold {width} values of x's dtype on its device")
    if not t.is_contiguous():
        t = t.contiguous()
    return t, t.data_ptr()


def _numbers(t: torch.Tensor, name: str, device: int, size: Optional[int] = None) -> torch.Tensor:
    """A vector of 64-bit integers."""
    if not isinstance(t, torch.Tensor) or t.get_device() != device or t.dtype is not torch.int64 or t.dim() != 1:
        raise ValueError(f"{name} must be a tensor of dtype torch.int64 with 1 dimension on the device of the states")
    if size is not None and t.shape[0] != size:
        raise ValueError(f"{name} must hold {size} values, got {t.shape[0]}")
    return t if t.is_contiguous() else t.contiguous()


def _stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def plaid_embedding(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """scale * table[ids] for a table [vocabulary, width] and ids [n] int64; zeros for an id outside the vocabulary."""
    dev = _states(table, "table")
    if _forward._current_level >= 0:
        _no_tangents(table=table)
    if _recording() and table.requires_grad:
        _not_recorded("plaid_embedding_backward", table=table)
    ids = _numbers(ids, "ids", dev)
    table, stride = _rows(table)
    vocabulary, width = table.shape
    n = ids.shape[0]
    out = table.new_empty((n, width))
    _p._check(_p.load_library().plaid_embedding(table.data_ptr(), stride, vocabulary, width, ids.data_ptr(), n, scale, out.data_ptr(), _DTYPES[table.dtype],
                                                dev, _stream(dev)))
    return out


def plaid_embedding_backward(d_out: torch.Tensor, ids: torch.Tensor, vocabulary: int, scale: float = 1.0,
                             add_to: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient [vocabulary, width] of plaid_embedding's table from that of its result, d_out [n, width]: dense, or added in place to
    `add_to`, which it then returns (a contiguous gradient of the same table from another use)."""
    dev = _states(d_out, "d_out")
    if _forward._current_level >= 0:
        _no_tangents(d_out=d_out, add_to=add_to)
    if _recording() and (d_out.requires_grad or add_to is not None):
        _not_recorded(None, d_out=d_out, add_to=add_to)
    ids = _numbers(ids, "ids", dev, d_out.shape[0])
    d_out, stride = _rows(d_out)
    n, width = d_out.shape
    if add_to is None:
        d_table = d_out.new_empty((vocabulary, width))
    else:
        d_table = _same(add_to, "add_to", d_out.dtype, (vocabulary, width), dev)
        if not d_table.is_contiguous():
            raise ValueError("add_to must be contiguous")
    lib = _p.load_library()
    need = ct.c_int64(0)
    _p._check(lib.plaid_embedding_backward_workspace(n, vocabulary, width, ct.byref(need)))
    work, ptr = _workspace(need.value, d_out.device)
    _p._check(lib.plaid_embedding_backward(d_out.data_ptr(), stride, vocabulary, width, ids.data_ptr(), n, scale, 0 if add_to is None else 1,
                                           d_table.data_ptr(), _DTYPES[d_out.dtype], ptr, need.value, dev, _stream(dev)))
    return d_table


def plaid_dropout(x: torch.Tensor, p: float, rng: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + dropout of x, any shape: an element is zero with the probability p (a multiple of 2^-16), else x / (1 - p).  rng [2] int64
    on x's device: a seed, and a number that no other call of the program has.  The gradient of x is the same call on the result's
    gradient, without a residual; the residual's is the result's."""
    dev = _states(x, "x", None)
    if _forward._current_level >= 0:
        _no_tangents(x=x, residual=residual)
    if _recording() and (x.requires_grad or residual is not None):
        _not_recorded("plaid_dropout", x=x, residual=residual)
    rng = _numbers(rng, "rng", dev, 2)
    if not x.is_contiguous():
        x = x.contiguous()
    other = None
    if residual is not None:
        residual = _same(residual, "residual", x.dtype, x.shape, dev).contiguous()
        other = residual.data_ptr()
    out = torch.empty_like(x)
    _p._check(_p.load_library().plaid_dropout(x.data_ptr(), other, x.numel(), p, rng.data_ptr(), out.data_ptr(), _DTYPES[x.dtype], dev, _stream(dev)))
    return out


def plaid_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                     return_statistics: bool = False):
    """Layer norm of the rows of x [rows, width], times weight [width], plus bias [width].  With return_statistics also what
    plaid_layer_norm_backward wants, each row's mean and 1 / sqrt(variance + eps), [rows, 2] float32."""
    dev = _states(x, "x")
    if _forward._current_level >= 0:
        _no_tangents(x=x, weight=weight, bias=bias)
    if _recording() and (x.requires_grad or weight is not None or bias is not None):
        _not_recorded("plaid_layer_norm_backward", x=x, weight=weight, bias=bias)
    x, stride = _rows(x)
    rows, width = x.shape
    weight, w = _parameter(weight, "weight", x, width, dev)
    bias, b = _parameter(bias, "bias", x, width, dev)
    out = torch.empty_like(x) if stride == width else x.new_empty((rows, width))
    statistics = x.new_empty((rows, 2), dtype=torch.float32) if return_statistics else None
    _p._check(_p.load_library().plaid_layer_norm(x.data_ptr(), stride, w, b, rows, width, eps, out.data_ptr(), None if statistics is None else statistics.data_ptr(),
                                                 _DTYPES[x.dtype], dev, _stream(dev)))
    return (out, statistics) if return_statistics else out


def plaid_layer_norm_backward(d_out: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], bias: Optional[torch.Tensor],
                              statistics: torch.Tensor):
    """(dx, dweight, dbias) of plaid_layer_norm from its statistics and the gradient d_out; None for a weight or bias that there is not."""
    dev = _states(x, "x")
    _same(d_out, "d_out", x.dtype, x.shape, dev)
    if _forward._current_level >= 0:
        _no_tangents(d_out=d_out, x=x, weight=weight, bias=bias, statistics=statistics)
    if _recording():
        _not_recorded(None, d_out=d_out, x=x, weight=weight, bias=bias, statistics=statistics)
    rows, width = x.shape
    weight, w = _parameter(weight, "weight", x, width, dev)
    bias, _ = _parameter(bias, "bias", x, width, dev)
    statistics = _same(statistics, "statistics", torch.float32, (rows, 2), dev).contiguous()
    x, stride = _rows(x)
    d_out, d_stride = _rows(d_out)
    dx = torch.empty_like(x) if stride == width else x.new_empty((rows, width))
    dweight = None if weight is None else torch.empty_like(weight)
    dbias = None if bias is None else torch.empty_like(bias)
    lib = _p.load_library()
    need = ct.c_int64(0)
    if weight is not None or bias is not None:
        _p._check(lib.plaid_layer_norm_backward_workspace(rows, width, ct.byref(need)))
    work, ptr = _workspace(need.value, x.device)
    _p._check(lib.plaid_layer_norm_backward(d_out.data_ptr(), d_stride, x.data_ptr(), stride, w, statistics.data_ptr(), rows, width, dx.data_ptr(),
                                            None if dweight is None else dweight.data_ptr(), None if dbias is None else dbias.data_ptr(), _DTYPES[x.dtype], ptr,
                                            need.value, dev, _stream(dev)))
    return dx, dweight, dbias


_PACKED = struct.Struct("2i2qf2P2q3P")  # plaid_token_loss's fields, as the C compiler lays them out


def _loss_args(hidden, weight, targets, scale, loss, lse) -> plaid_token_loss:
    """hidden, weight: what _aligned_rows gave."""
    (h, h_stride), (w, w_stride) = hidden, weight
    return plaid_token_loss.from_buffer_copy(_PACKED.pack(_DTYPES[h.dtype], h.shape[1], h.shape[0], w.shape[0], scale, h.data_ptr(), w.data_ptr(), h_stride, w_stride,
                                                          targets.data_ptr(), 0 if loss is None else loss.data_ptr(), 0 if lse is None else lse.data_ptr()))


def _loss_inputs(hidden, weight, targets):
    dev = _states(hidden, "hidden")
    if _states(weight, "weight") != dev or weight.dtype is not hidden.dtype or weight.shape[1] != hidden.shape[1]:
        raise ValueError("hidden and weight must have rows of one width, one dtype and one device")
    targets = _numbers(targets, "targets", dev, hidden.shape[0])
    return _aligned_rows(hidden), _aligned_rows(weight), targets


def plaid_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, scale: float = 1.0, return_lse: bool = False):
    """The negative logarithm of each target's probability under softmax(scale * hidden @ weight.T): hidden [rows, width], weight
    [vocabulary, width], targets [rows] int64 -> [rows] float32, zero for a target outside the vocabulary.  With return_lse also what
    plaid_cross_entropy_backward wants, the logarithm of the softmax's sum as two numbers to be added, [rows, 2] float32."""
    rows, table, targets = _loss_inputs(hidden, weight, targets)
    if _forward._current_level >= 0:
        _no_tangents(hidden=hidden, weight=weight)
    if _recording() and (hidden.requires_grad or weight.requires_grad):
        _not_recorded("plaid_cross_entropy_backward", hidden=hidden, weight=weight)
    dev = hidden.get_device()
    n = hidden.shape[0]
    loss = hidden.new_empty(n, dtype=torch.float32)
    lse = hidden.new_empty((n, 2), dtype=torch.float32) if return_lse else None
    lib = _p.load_library()
    a = _loss_args(rows, table, targets, scale, loss, lse)
    need = ct.c_int64(0)
    _p._check(lib.plaid_cross_entropy_workspace(ct.byref(a), 0, ct.byref(need)))
    work, ptr = _workspace(need.value, hidden.device)
    _p._check(lib.plaid_cross_entropy(ct.byref(a), ptr, need.value, dev, _stream(dev)))
    return (loss, lse) if return_lse else loss


def plaid_cross_entropy_backward(d_loss: torch.Tensor, hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                                 scale: float = 1.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """(d_hidden, d_weight) of plaid_cross_entropy from its lse and the gradient of its result, d_loss [rows] float32 (an expanded single
    number is taken as it is)."""
    rows, table, targets = _loss_inputs(hidden, weight, targets)
    dev, n = hidden.get_device(), hidden.shape[0]
    if _forward._current_level >= 0:
        _no_tangents(d_loss=d_loss, hidden=hidden, weight=weight, lse=lse)
    if _recording():
        _not_recorded(None, d_loss=d_loss, hidden=hidden, weight=weight, lse=lse)
    if _same(d_loss, "d_loss", torch.float32, (n,), dev).stride(0) not in (0, 1):
        d_loss = d_loss.contiguous()
    lse = _same(lse, "lse", torch.float32, (n, 2), dev).contiguous()
    d_hidden = hidden.new_empty(hidden.shape)
    d_weight = hidden.new_empty(weight.shape)
    lib = _p.load_library()
    a = _loss_args(rows, table, targets, scale, None, lse)
    need = ct.c_int64(0)
    _p._check(lib.plaid_cross_entropy_workspace(ct.byref(a), 1, ct.byref(need)))
    work, ptr = _workspace(need.value, hidden.device)
    _p._check(lib.plaid_cross_entropy_backward(ct.byref(a), d_loss.data_ptr(), d_loss.stride(0) if n > 1 else 1, d_hidden.data_ptr(), d_weight.data_ptr(), ptr, need.value,
                                               dev, _stream(dev)))
    return d_hidden, d_weight
