"""The norms around a block of libsscater.so (argument marshalling only), over rows
of cells or tokens.  They form no gradients: where one would be wanted they refuse
the call."""
from __future__ import annotations

from functools import lru_cache
from typing import Optional

from . import engine as E
from . import tokens as T
from .engine import lib

GATES = {None: 0, "none": 0, "silu": 3, "sigmoid": 4}

# the descriptions of the last calls' sizes (making one takes 1.2 us, finding it 0.2)
_spec = lru_cache(256)(E.NormSpec)


def _width(t, name: str, dtype, index: int, width: int):
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != index or t.dim() != 1 or t.shape[0] != width:
        T._require(t, name, dtype, index, (width,))
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.requires_grad:
        T._want_gradient()
    return t.data_ptr()


def _rows(t, name: str, dtype, index: int, shape, width: int) -> int:
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        T._require(t, name, dtype, index, shape)
    if t.requires_grad:
        T._want_gradient()
    return width if t.is_contiguous() else T._row_stride(t, name, width)


def _gate(gate, dtype, index: int, shape, width: int, rows: int):
    """The gate's row stride, and how many rows share one of its rows: its shape is
    the rows' without some of the axes before the last."""
    lead = gate.dim() - 1
    if lead < 0 or lead > len(shape) - 1 or gate.shape[:-1] != shape[:lead] or gate.shape[-1] != width:
        raise ValueError(f"gate must be {tuple(shape)} or that without axes before the last, not {tuple(gate.shape)}")
    n = gate.numel() // width
    return _rows(gate, "gate", dtype, index, gate.shape, width), max(rows // n if n else 1, 1)


def _call(x, block, block_norm, block_weight, block_bias, gate, activation, scale, weight, bias, eps, center, total, y,
          stream):
    """One library call; total and y (only with a weight) are made unless they are given, and returned."""
    act = GATES.get(activation, -1)
    if act < 0:
        raise ValueError(f"activation of a gate must be one of {sorted(k for k in GATES if k)}")
    if gate is None and act:
        raise ValueError("an activation without a gate")
    dtype, shape, index = block.dtype, block.shape, block.get_device()
    width = shape[-1]
    rows = block.numel() // width
    ldb = _rows(block, "block" if x is not None else "x", dtype, index, shape, width)
    ldx = width if x is None else _rows(x, "x", dtype, index, shape, width)
    ldg, shared = (width, 1) if gate is None else _gate(gate, dtype, index, shape, width, rows)
    if total is None:
        total, lds = block.new_empty(shape), width
    else:
        lds = _rows(total, "out" if x is None else "total", dtype, index, shape, width)
    if y is not None:
        ldy = _rows(y, "out", dtype, index, shape, width)
        if y.data_ptr() == total.data_ptr() and rows:
            raise ValueError("total and out must be two tensors")
    else:
        y, ldy = None if weight is None else block.new_empty(shape), width
    spec = _spec(rows, shared, width, T._KINDS[dtype], 1 if center else 0, 1 if block_norm else 0, act, T._number(eps), ldx,
                 ldb, ldg, lds, ldy)
    T._launch(lib().sscater_norm, "sscater_norm", index, stream,
              (x, block, gate, total, y, block_weight, block_bias, scale, weight, bias), spec,
              None if x is None else x.data_ptr(), block.data_ptr(), _width(block_weight, "block_weight", dtype, index, width),
              _width(block_bias, "block_bias", dtype, index, width), None if gate is None else gate.data_ptr(),
              _width(scale, "scale", dtype, index, width), _width(weight, "weight", dtype, index, width),
              _width(bias, "bias", dtype, index, width), total.data_ptr(), None if y is None else y.data_ptr())
    return total, y


def _tensor(t, name: str) -> None:
    if T.torch is None:
        T._bind()
    if t.dtype not in T._KINDS:
        raise ValueError(f"float32 or bfloat16 tensors, not {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a cuda tensor")
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{name} must be [..., width], of at least one value")


def norm(x, weight=None, bias=None, eps: float = 1e-6, center: bool = False, gate=None,
         activation: Optional[str] = None, out=None, stream=None):
    """act(gate) * (N(x) * weight + bias), N(x) = x / sqrt(mean(x^2) + eps), of x less
    its mean with center.  x [..., width] (float32 or bfloat16, its rows evenly apart),
    weight and bias [width]; gate of x's shape, or of it without some of the axes before
    the last (one for each image of a batch, say); activation none, silu or sigmoid.
    out may be x, or a gate of its shape, and must not overlap the other operands."""
    _tensor(x, "x")
    return _call(None, x, True, weight, bias, gate, activation, None, None, None, eps, center, out, None, stream)[0]


def add_norm(x, block, weight=None, bias=None, *, block_weight=None, block_bias=None, gate=None,
             activation: Optional[str] = None, scale=None, eps: float = 1e-6, center: bool = False, total=None, out=None,
             stream=None):
    """A block's output into the residual stream, and the next block's input:
    total = x + scale * act(gate) * P(block) and out = N(total) * weight + bias, both
    returned.  P is the norm with block_weight and block_bias (without block_weight it
    is left out), N the one of norm(); without weight, out is None.  x, block, total and
    out [..., width], gate as for norm(), the rest [width].  total may be x or block, out
    too (not both the same); otherwise they overlap nothing."""
    _tensor(block, "block")
    if weight is None and (bias is not None or out is not None):
        raise ValueError("bias and out come with weight")
    if block_weight is None and block_bias is not None:
        raise ValueError("block_bias comes with block_weight")
    return _call(x, block, block_weight is not None, block_weight, block_bias, gate, activation, scale, weight, bias, eps,
                 center, total, out, stream)
