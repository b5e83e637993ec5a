"""Attention of one set of tokens to another in libsscater.so (argument marshalling
only).  It forms no gradients: where one would be wanted it refuses the call."""
from __future__ import annotations

import ctypes
from functools import lru_cache
from typing import Optional

from . import engine as E
from . import tokens as T
from .engine import _check, lib


def _heads(t, name: str, dtype, index: int, dims: int) -> int:
    """The row stride of [..., heads, head_dim]: heads one behind the other, rows
    evenly apart, on 16-byte boundaries."""
    if t.dtype is not dtype or t.get_device() != index:
        T._require(t, name, dtype, index)
    shape, stride = t.shape, t.stride()
    if len(shape) != dims or 0 in shape[-2:]:
        raise ValueError(f"{name} must have {dims} axes as q has, and at least one head")
    n, heads, dim = shape[-3:]
    width = ld = heads * dim
    if stride[-1] != 1 and dim > 1 or stride[-2] != dim and heads > 1:
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    batch = shape[0] if dims == 4 else 1
    if n > 0 and batch > 0:
        if n > 1:
            ld = stride[-3]
            if batch > 1 and stride[0] != n * ld:
                raise ValueError(f"{name}: its rows must lie evenly apart")
        elif batch > 1:
            ld = stride[0]
        if ld < width:
            raise ValueError(f"{name}: its rows overlap")
        if t.data_ptr() % 16 or ld * t.element_size() % 16:
            raise ValueError(f"{name}: its rows must lie on 16-byte boundaries")
    if t.requires_grad:
        T._want_gradient()
    return ld


def _describe(masked: int, *fields):
    """A call's description, and the bytes of its workspace."""
    spec, need = E.CrossSpec(*fields), ctypes.c_size_t()
    _check(lib().sscater_cross_workspace(spec, masked, need), "sscater_cross_workspace")
    return spec, need.value


# of sizes alone, without addresses (2.6 us to make, 0.2 to find)
_described = lru_cache(256)(_describe)


def cross_attend(q, k, v, mask=None, q_start=None, k_start=None, max_q: Optional[int] = None,
                 max_k: Optional[int] = None, scale: Optional[float] = None, out=None, stream=None, rounded: bool = False):
    """Attention of queries to the keys and values of another set of tokens (objects
    to a map's cells): softmax(scale * q k^T) v over the visible keys; zeros where a
    sequence has none.

    q [batch, queries, q_heads, head_dim] and k, v [batch, keys, kv_heads, head_dim]
    (without the batch axis: one sequence), mask [batch, keys] of bool or uint8, true
    where a key is visible (None: everywhere; what k and v hold elsewhere does not
    matter).  Sequences of different lengths: q [queries, q_heads, head_dim], k and v
    [keys, kv_heads, head_dim], mask [keys], with q_start and k_start (int32 cuda
    tensors [batch + 1], sequence b being rows start[b] to start[b + 1] - 1) and the most
    of one sequence, max_q and max_k, where they are known.  float32 or bfloat16,
    head_dim 32, 64 or 128, q_heads a multiple of kv_heads; rows may be columns of a
    projection's, evenly apart and on 16-byte boundaries.  scale: 1 / sqrt(head_dim)
    unless given.  out: q's shape, contiguous, overlapping no operand.  rounded
    (bfloat16, where a sequence may bring more than 32 rows, max_q * q_heads / kv_heads):
    probabilities rounded to bfloat16 for the product with the values, an error as large
    as the output's rounding, in some seven tenths of the time."""
    if T.torch is None:
        T._bind()
    dtype = q.dtype
    kind = T._KINDS.get(dtype, -1)
    if kind < 0:
        raise ValueError(f"float32 or bfloat16 tensors, not {dtype}")
    index, dims = q.get_device(), q.dim()
    if index < 0:
        raise ValueError("q must be a cuda tensor")
    if dims not in (3, 4):
        raise ValueError("q must be [queries, q_heads, head_dim] or [batch, queries, q_heads, head_dim]")
    ldq = _heads(q, "q", dtype, index, dims)
    ldk, ldv = _heads(k, "k", dtype, index, dims), _heads(v, "v", dtype, index, dims)
    heads, dim = q.shape[-2], q.shape[-1]
    if k.shape != v.shape or k.shape[-1] != dim or heads % k.shape[-2]:
        raise ValueError("k and v must be of one shape, of q's head_dim and of heads that divide q's")
    if dim not in (32, 64, 128):
        raise ValueError("head_dim 32, 64 or 128")
    if (q_start is None) != (k_start is None):
        raise ValueError("q_start and k_start come together")
    if q_start is not None:
        if dims != 3:
            raise ValueError("q_start and k_start come with q, k and v of three axes")
        batch, queries, keys = q_start.numel() - 1, q.shape[0], k.shape[0]
        if batch < 1:
            raise ValueError("q_start and k_start must be [batch + 1]")
        at = [T._dense(t, name, T.torch.int32, index, (batch + 1,)) for name, t in (("q_start", q_start), ("k_start", k_start))]
        max_q, max_k = queries if max_q is None else int(max_q), keys if max_k is None else int(max_k)
    else:
        if max_q is not None or max_k is not None:
            raise ValueError("max_q and max_k come with q_start and k_start")
        if dims == 4 and k.shape[0] != q.shape[0]:
            raise ValueError("q, k and v must be of one batch")
        batch = q.shape[0] if dims == 4 else 1
        max_q, max_k, at = q.shape[-3], k.shape[-3], (None, None)
        queries, keys = batch * max_q, batch * max_k
    if mask is not None:
        if mask.dtype not in (T.torch.bool, T.torch.uint8):
            raise ValueError(f"mask must be bool or uint8, not {mask.dtype}")
        T._dense(mask, "mask", mask.dtype, index, k.shape[:-2])
    if out is None:
        out = q.new_empty(q.shape)
    elif T._dense(out, "out", dtype, index, q.shape) % 16:
        raise ValueError("out must be on a 16-byte boundary")
    elif out.requires_grad:
        T._want_gradient()
    if queries == 0:
        return out
    spec, need = (_described if q_start is None else _describe)(
        0 if mask is None else 1, kind, batch, heads, k.shape[-2], dim, queries, keys, max_q, max_k,
        dim ** -0.5 if scale is None else T._number(scale), ldq, ldk, ldv, *at, 1 if rounded else 0)
    work = q.new_empty(need, dtype=T.torch.uint8) if need else None
    T._launch(lib().sscater_cross_attend, "sscater_cross_attend", index, stream, (q, k, v, mask, q_start, k_start, out, work),
              spec, q.data_ptr(), k.data_ptr(), v.data_ptr(), None if mask is None else mask.data_ptr(), out.data_ptr(),
              None if work is None else work.data_ptr(), need)
    return out
