"""Binding of the reader's operators (include/plaid.h): block tables, the paged cache in four bits, attention over it, cross
attention and its gradients.

Like `plaid.py` this only marshals: it checks tensors, allocates outputs and workspaces from torch's allocator and hands over
torch's current stream of the tensors' device.  Nothing is kept from one call for the next.
"""
from __future__ import annotations

import ctypes as ct
import struct
from typing import Optional, Tuple

import torch

from . import plaid as _p

PLAID_BF16, PLAID_FP16 = 0, 1
_DTYPES = {torch.bfloat16: PLAID_BF16, torch.float16: PLAID_FP16}
_BLOCK_SIZES = (16, 32, 64, 128, 256)


class plaid_paged_cache(ct.Structure):
    _fields_ = [("data", ct.c_void_p), ("num_blocks", ct.c_int64), ("block_size", ct.c_int32), ("kv_heads", ct.c_int32),
                ("head_dim", ct.c_int32), ("dtype", ct.c_int32)]


class plaid_attention(ct.Structure):
    _fields_ = ([(n, ct.c_int32) for n in ("dtype", "n", "heads", "kv_heads", "head_dim")] + [("scale", ct.c_float)]
                + [(n, ct.c_int64) for n in ("num_queries", "num_keys")] + [(n, ct.c_void_p) for n in ("q", "k", "v", "key_bias")]
                + [(n, ct.c_int64) for n in ("q_token_stride", "q_head_stride", "k_token_stride", "k_head_stride", "v_token_stride", "v_head_stride")]
                + [(n, ct.c_void_p) for n in ("q_offsets", "k_offsets", "out", "lse")])


def declare(lib: ct.CDLL) -> None:
    """Argument types of the reader's functions."""
    P, i32, i64 = ct.c_void_p, ct.c_int32, ct.c_int64
    attention, cache, out64 = ct.POINTER(plaid_attention), ct.POINTER(plaid_paged_cache), ct.POINTER(i64)
    lib.plaid_block_tables.argtypes = [P, P, i32, P, i64, i32, P, i32, i32, P, P, P, P, i64, P, P, i64, ct.c_int, P]
    lib.plaid_block_tables_workspace.argtypes = [i32, i64, out64]
    lib.plaid_cache_write.argtypes = [cache, P, P, i64, i64, i64, i64, P, i64, ct.c_int, P]
    lib.plaid_cache_read.argtypes = [cache, P, i64, P, P, ct.c_int, P]
    lib.plaid_cached_attention.argtypes = [attention, cache, P, i64, i32, P, i32, P, i64, ct.c_int, P]
    lib.plaid_cached_attention_workspace.argtypes = [attention, i32, i32, out64]
    lib.plaid_cross_attention.argtypes = [attention, P, i64, ct.c_int, P]
    lib.plaid_cross_attention_backward.argtypes = [attention, P, P, P, P, P, P, i64, ct.c_int, P]
    lib.plaid_cross_attention_workspace.argtypes = [attention, i32, out64]


def _is(t: torch.Tensor, name: str, dtype, dim: int, device: Optional[torch.device] = None) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or t.dim() != dim:
        raise ValueError(f"{name} must be a CUDA tensor of dtype {dtype} with {dim} dimension(s)")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on another device than the other tensors")
    return t


def _vector(t: torch.Tensor, name: str, dtype, device: torch.device, size: Optional[int] = None) -> torch.Tensor:
    _is(t, name, dtype, 1, device)
    if size is not None and t.shape[0] != size:
        raise ValueError(f"{name} must hold {size} values, got {t.shape[0]}")
    return t.contiguous()


def _rows(t: torch.Tensor) -> Tuple[torch.Tensor, int, int]:
    """The tensor itself where the kernels can read its strides, else a contiguous copy, and its strides of tokens and heads."""
    n, heads, dim = t.shape
    token, head, one = t.stride()
    if n < 2:
        token = heads * dim
    if heads < 2:
        head = dim
    if one != 1 or token % 8 or head % 8 or token >= 1 << 24 or head >= 1 << 24 or t.data_ptr() % 16:
        if t.numel():
            t = t.contiguous() if not t.is_contiguous() else t.clone(memory_format=torch.contiguous_format)
        token, head = heads * dim, dim
    return t, token, head


def _like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t) if t.is_contiguous() else torch.empty_like(t, memory_format=torch.contiguous_format)


def _workspace(bytes_: int, device: torch.device):
    """(tensor that the caller holds until its launches are made, its address)"""
    if bytes_ == 0:
        return None, None
    w = torch.empty(bytes_, dtype=torch.uint8, device=device)
    return w, w.data_ptr()


def _where(device: torch.device) -> Tuple[int, int]:
    """Ordinal of a device and torch's current stream there."""
    i = device.index or 0
    return i, torch._C._cuda_getCurrentRawStream(i)


class PagedCache:
    """Keys and values of a paged cache in four bits a value.

    `data` is a contiguous uint8 tensor [num_blocks, kv_heads, block_size * head_dim * 17 / 16], laid out as include/plaid.h says;
    `dtype` (torch.bfloat16 or torch.float16) is the type that is written and read.  The object holds the tensor, nothing else."""

    def __init__(self, data: torch.Tensor, block_size: int, head_dim: int, dtype: torch.dtype):
        _is(data, "data", torch.uint8, 3)
        if dtype not in _DTYPES:
            raise ValueError("the cache's dtype must be torch.bfloat16 or torch.float16")
        if block_size not in _BLOCK_SIZES:
            raise ValueError(f"block_size must be one of {_BLOCK_SIZES}")
        if head_dim not in (64, 128) or data.shape[2] * 16 != block_size * head_dim * 17:
            raise ValueError("head_dim must be 64 or 128 and data.shape[2] block_size * head_dim * 17 / 16")
        if not data.is_contiguous() or data.data_ptr() % 16:
            raise ValueError("data must be contiguous and 16-byte aligned")
        self.data, self.block_size, self.head_dim, self.dtype = data, int(block_size), int(head_dim), dtype
        self.num_blocks, self.kv_heads = data.shape[0], data.shape[1]

    @classmethod
    def empty(cls, num_blocks: int, block_size: int, kv_heads: int, head_dim: int, dtype: torch.dtype, device="cuda:0") -> "PagedCache":
        """A cache of zeros."""
        region = int(block_size) * int(head_dim) * 17 // 16
        return cls(torch.zeros((num_blocks, kv_heads, region), dtype=torch.uint8, device=device), block_size, head_dim, dtype)

    def _view(self) -> plaid_paged_cache:
        return plaid_paged_cache(self.data.data_ptr(), self.num_blocks, self.block_size, self.kv_heads, self.head_dim, _DTYPES[self.dtype])


def plaid_block_tables(lengths: torch.Tensor, added: torch.Tensor, table: torch.Tensor, free_blocks: torch.Tensor, block_size: int,
                       capacity: int):
    """Hands blocks of a paged cache to requests that hold `lengths` [n] tokens and get `added` [n] more (int32), in place in
    `table` [n, max_blocks] int32; `capacity`: room for new tokens, normally their number.  Returns (offsets [n+1] int64, totals
    [n] int32, positions [capacity] int32, slots [capacity] int64, blocks_wanted [1] int64).  More blocks wanted than
    `free_blocks` holds, or a full row of the table, leaves slots of -1."""
    dev = _is(lengths, "lengths", torch.int32, 1).device
    n = lengths.shape[0]
    lengths = lengths.contiguous()
    added = _vector(added, "added", torch.int32, dev, n)
    free_blocks = _vector(free_blocks, "free_blocks", torch.int32, dev)
    _is(table, "table", torch.int32, 2, dev)
    if table.shape[0] != n or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must have a row for each request and contiguous rows")
    lib, capacity = _p.load_library(), int(capacity)
    need = ct.c_int64(0)
    _p._check(lib.plaid_block_tables_workspace(n, capacity, ct.byref(need)))
    room = max(capacity, 0)
    offsets = torch.empty(n + 1, dtype=torch.int64, device=dev)
    totals = torch.empty_like(lengths)
    positions = torch.empty(room, dtype=torch.int32, device=dev)
    slots = torch.empty(room, dtype=torch.int64, device=dev)
    wanted = torch.empty(1, dtype=torch.int64, device=dev)
    work, ptr = _workspace(need.value, dev)
    _p._check(lib.plaid_block_tables(lengths.data_ptr(), added.data_ptr(), n, table.data_ptr(), table.stride(0) if n > 1 else table.shape[1],
                                     table.shape[1], free_blocks.data_ptr(), free_blocks.shape[0], int(block_size), offsets.data_ptr(),
                                     totals.data_ptr(), positions.data_ptr(), slots.data_ptr(), capacity, wanted.data_ptr(), ptr, need.value,
                                     *_where(dev)))
    return offsets, totals, positions, slots, wanted


def plaid_cache_write(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """Writes k and v [tokens, kv_heads, head_dim] of the cache's dtype to `slots` [tokens] int64 (negative: left out)."""
    dev = cache.data.device
    shape = (slots.shape[0], cache.kv_heads, cache.head_dim)
    for name, t in (("k", k), ("v", v)):
        if tuple(_is(t, name, cache.dtype, 3, dev).shape) != shape:
            raise ValueError(f"{name} must have the shape {shape}, got {tuple(t.shape)}")
    slots = _vector(slots, "slots", torch.int64, dev)
    k, k_token, k_head = _rows(k)
    v, v_token, v_head = _rows(v)
    _p._check(_p.load_library().plaid_cache_write(ct.byref(cache._view()), k.data_ptr(), v.data_ptr(), k_token, k_head, v_token, v_head,
                                                  slots.data_ptr(), slots.shape[0], *_where(dev)))


def plaid_cache_read(cache: PagedCache, slots: torch.Tensor):
    """(k, v) [tokens, kv_heads, head_dim] that `slots` [tokens] int64 hold; zeros for a slot outside the cache."""
    dev = cache.data.device
    slots = _vector(slots, "slots", torch.int64, dev)
    k = torch.empty((slots.shape[0], cache.kv_heads, cache.head_dim), dtype=cache.dtype, device=dev)
    v = torch.empty_like(k)
    _p._check(_p.load_library().plaid_cache_read(ct.byref(cache._view()), slots.data_ptr(), slots.shape[0], k.data_ptr(), v.data_ptr(),
                                                 *_where(dev)))
    return k, v


_PACKED = struct.Struct("5if2q4P6q4P")  # plaid_attention's fields: half the time of the structure's own constructor


def _attention(q, k, v, key_bias, q_offsets, k_offsets, kv_heads, scale, out, lse) -> plaid_attention:
    """q, k and v: what _rows gave (k and v None over a cache)."""
    q, q_token, q_head = q
    tokens, heads, head_dim = q.shape
    keys = k_ptr = v_ptr = k_token = k_head = v_token = v_head = k_off = 0
    if k is not None:
        (k, k_token, k_head), (v, v_token, v_head) = k, v
        keys, k_ptr, v_ptr, k_off = k.shape[0], k.data_ptr(), v.data_ptr(), k_offsets.data_ptr()
    return plaid_attention.from_buffer_copy(_PACKED.pack(
        _DTYPES[q.dtype], q_offsets.shape[0] - 1, heads, kv_heads, head_dim, head_dim ** -0.5 if scale is None else float(scale), tokens, keys,
        q.data_ptr(), k_ptr, v_ptr, 0 if key_bias is None else key_bias.data_ptr(), q_token, q_head, k_token, k_head, v_token, v_head,
        q_offsets.data_ptr(), k_off, out.data_ptr(), 0 if lse is None else lse.data_ptr()))


def _check_heads(q: torch.Tensor, kv_heads: int, head_dim: int) -> None:
    if q.shape[2] != head_dim or head_dim not in (64, 128):
        raise ValueError(f"head_dim must be 64 or 128 and the same for queries and keys, got {q.shape[2]} and {head_dim}")
    if kv_heads < 1 or q.shape[1] < 1 or q.shape[1] % kv_heads:
        raise ValueError(f"{q.shape[1]} query heads are no multiple of {kv_heads} key heads")


def _check_queries(q: torch.Tensor) -> None:
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dtype not in _DTYPES or q.dim() != 3:
        raise ValueError("q must be a CUDA tensor [tokens, heads, head_dim] of dtype torch.bfloat16 or torch.float16")


def plaid_cached_attention(q: torch.Tensor, cache: PagedCache, table: torch.Tensor, lengths: torch.Tensor, q_offsets: torch.Tensor,
                           scale: Optional[float] = None, causal: bool = True, return_lse: bool = False):
    """Attention of q [tokens, heads, head_dim] over a paged cache: request r's queries are rows q_offsets[r] .. q_offsets[r+1]-1
    (int64 [n+1]), its keys the lengths[r] (int32) tokens that table[r] ([n, max_blocks] int32) leads to.  causal: the queries are
    the request's last tokens, each sees what is not after it.  scale: head_dim ** -0.5 by default.  Returns out like q, with
    return_lse also the logarithm of the softmax's sum as two numbers to be added, [tokens, heads, 2] float32.  It has no gradient:
    what the cache holds is rounded."""
    _check_queries(q)
    dev = q.device
    if cache.data.device != dev or q.dtype != cache.dtype:
        raise ValueError("q and the cache must have one device and dtype")
    _check_heads(q, cache.kv_heads, cache.head_dim)
    n = _is(lengths, "lengths", torch.int32, 1, dev).shape[0]
    lengths = lengths.contiguous()
    q_offsets = _vector(q_offsets, "q_offsets", torch.int64, dev, n + 1)
    _is(table, "table", torch.int32, 2, dev)
    if table.shape[0] != n:
        raise ValueError("table must have a row for each request")
    if table.shape[1] > 1 and table.stride(1) != 1:
        table = table.contiguous()
    rows = _rows(q)
    out = _like(q)
    lse = torch.empty(q.shape[:2] + (2,), dtype=torch.float32, device=dev) if return_lse else None
    lib = _p.load_library()
    a = _attention(rows, None, None, None, q_offsets, None, cache.kv_heads, scale, out, lse)
    need = ct.c_int64(0)
    _p._check(lib.plaid_cached_attention_workspace(ct.byref(a), table.shape[1], cache.block_size, ct.byref(need)))
    work, ptr = _workspace(need.value, dev)
    _p._check(lib.plaid_cached_attention(ct.byref(a), ct.byref(cache._view()), table.data_ptr(), table.stride(0) if n > 1 else table.shape[1],
                                         table.shape[1], lengths.data_ptr(), 1 if causal else 0, ptr, need.value, *_where(dev)))
    return (out, lse) if return_lse else out


def _cross_inputs(q, k, v, q_offsets, k_offsets, key_bias):
    _check_queries(q)
    dev = q.device
    for name, t in (("k", k), ("v", v)):
        _is(t, name, q.dtype, 3, dev)
    if k.shape != v.shape:
        raise ValueError("k and v must have one shape")
    _check_heads(q, k.shape[1], k.shape[2])
    n = _is(q_offsets, "q_offsets", torch.int64, 1, dev).shape[0] - 1
    q_offsets = q_offsets.contiguous()
    k_offsets = _vector(k_offsets, "k_offsets", torch.int64, dev, n + 1)
    if key_bias is not None:
        key_bias = _vector(key_bias, "key_bias", q.dtype, dev, k.shape[0])
    return _rows(q), _rows(k), _rows(v), q_offsets, k_offsets, key_bias


def _no_autograd(**tensors) -> None:
    """The calls are not recorded: where one would be differentiated through, its result would be cut off without a word."""
    if torch.is_grad_enabled():
        for name, t in tensors.items():
            if t is not None and t.requires_grad:
                raise ValueError(f"{name} requires a gradient, which this call does not record: call it in torch.no_grad(), or in a "
                                 "torch.autograd.Function whose backward calls plaid_cross_attention_backward")


def plaid_cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor, k_offsets: torch.Tensor,
                          key_bias: Optional[torch.Tensor] = None, scale: Optional[float] = None, return_lse: bool = False):
    """Attention of q [tokens, heads, head_dim] to states of another length, k and v [keys, kv_heads, head_dim], both packed:
    request r owns rows q_offsets[r] .. q_offsets[r+1]-1 and keys k_offsets[r] .. k_offsets[r+1]-1 (int64 [n+1]).  key_bias [keys]
    of q's dtype is added to the scores; -inf takes a key out.  Returns out like q (rows outside every request are not written),
    with return_lse also the two numbers a row that plaid_cross_attention_backward wants.  Not recorded by autograd: inputs that
    require a gradient are refused where it is enabled (examples/reader.py has the torch.autograd.Function of both calls)."""
    rows, keys, values, q_offsets, k_offsets, key_bias = _cross_inputs(q, k, v, q_offsets, k_offsets, key_bias)
    _no_autograd(q=q, k=k, v=v, key_bias=key_bias)
    dev = q.device
    out = _like(q)
    lse = torch.empty(q.shape[:2] + (2,), dtype=torch.float32, device=dev) if return_lse else None
    lib = _p.load_library()
    a = _attention(rows, keys, values, key_bias, q_offsets, k_offsets, k.shape[1], scale, out, lse)
    need = ct.c_int64(0)
    _p._check(lib.plaid_cross_attention_workspace(ct.byref(a), 0, ct.byref(need)))
    work, ptr = _workspace(need.value, dev)
    _p._check(lib.plaid_cross_attention(ct.byref(a), ptr, need.value, *_where(dev)))
    return (out, lse) if return_lse else out


def plaid_cross_attention_backward(d_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                                   q_offsets: torch.Tensor, k_offsets: torch.Tensor, key_bias: Optional[torch.Tensor] = None,
                                   scale: Optional[float] = None):
    """(dq, dk, dv, dbias) of plaid_cross_attention, from its outputs out and lse and the gradient d_out; contiguous, dbias None
    without key_bias.  Rows outside every request are not written."""
    rows, keys, values, q_offsets, k_offsets, key_bias = _cross_inputs(q, k, v, q_offsets, k_offsets, key_bias)
    dev = q.device
    for name, t in (("d_out", d_out), ("out", out)):
        if _is(t, name, q.dtype, 3, dev).shape != q.shape:
            raise ValueError(f"{name} must have q's shape")
    _is(lse, "lse", torch.float32, 3, dev)
    if lse.shape != q.shape[:2] + (2,):
        raise ValueError("lse must be what plaid_cross_attention returned")
    whole = lambda t: t if t.is_contiguous() and t.data_ptr() % 16 == 0 else t.clone(memory_format=torch.contiguous_format)  # noqa: E731
    d_out, out, lse = whole(d_out), whole(out), whole(lse)
    dq = _like(q)
    dk = _like(k)
    dv = _like(k)
    dbias = torch.empty(k.shape[:1], dtype=q.dtype, device=dev) if key_bias is not None else None
    lib = _p.load_library()
    a = _attention(rows, keys, values, key_bias, q_offsets, k_offsets, k.shape[1], scale, out, lse)
    need = ct.c_int64(0)
    _p._check(lib.plaid_cross_attention_workspace(ct.byref(a), 1, ct.byref(need)))
    work, ptr = _workspace(need.value, dev)
    _p._check(lib.plaid_cross_attention_backward(ct.byref(a), d_out.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                                 None if dbias is None else dbias.data_ptr(), ptr, need.value, *_where(dev)))
    return dq, dk, dv, dbias
