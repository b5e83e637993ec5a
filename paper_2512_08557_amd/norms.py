"""The norms around a block of libsscater.so (argument marshalling only), over rows
of cells or tokens.  They form no gradients: where one would be wanted they refuse
the call."""
from __future__ import annotations

from typing import Optional

from . import engine as E
from . import tokens as T
from .engine import lib

GATES = {None: 0, "none": 0, "silu": 3, "sigmoid": 4}


def _width(t, name: str, dtype, index: int, width: int):
    T._require(t, name, dtype, index, (width,))
    if width > 1 and t.stride(0) != 1:
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _gate(gate, activation, x, dtype, index: int, rows: int):
    """The gate's row stride, and how many rows of x share one of its rows: its
    shape is x's without some of the axes before the last."""
    lead = gate.dim() - 1
    if lead < 0 or lead > x.dim() - 1 or gate.shape[:-1] != x.shape[:lead] or gate.shape[-1] != x.shape[-1]:
        raise ValueError(f"gate must be {tuple(x.shape)} or that without axes before the last, not {tuple(gate.shape)}")
    T._require(gate, "gate", dtype, index)
    n = gate.numel() // x.shape[-1]
    return T._row_stride(gate, "gate", x.shape[-1]), rows // n if n else 1


def _call(x, block, block_norm, block_weight, block_bias, gate, activation, scale, weight, bias, eps, center, total, y,
          stream) -> None:
    act = GATES.get(activation, -1)
    if act < 0:
        raise ValueError(f"activation of a gate must be one of {sorted(k for k in GATES if k)}")
    if gate is None and act:
        raise ValueError("an activation without a gate")
    dtype, shape, index = block.dtype, block.shape, block.get_device()
    width = shape[-1]
    rows = block.numel() // width
    stride = {"block": T._row_stride(block, "block" if x is not None else "x", width)}
    for name, t in (("x", x), ("total", total), ("out", y)):
        if t is not None:
            stride[name] = T._row_stride(T._require(t, name, dtype, index, shape), name, width)
    shared = 1
    if gate is not None:
        stride["gate"], shared = _gate(gate, activation, block, dtype, index, rows)
    vectors = (block_weight, block_bias, scale, weight, bias)
    at = [None if t is None else _width(t, name, dtype, index, width)
          for name, t in zip(("block_weight", "block_bias", "scale", "weight", "bias"), vectors)]
    for t in (x, block, gate) + vectors:
        if t is not None and t.requires_grad:
            T._want_gradient()
    spec = E.NormSpec(rows, max(shared, 1), width, T._KINDS[dtype], 1 if center else 0, 1 if block_norm else 0, act, eps,
                      stride.get("x", width), stride["block"], stride.get("gate", width), stride.get("total", width),
                      stride.get("out", width))
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    T._launch(lib().sscater_norm, "sscater_norm", index, stream, (x, block, gate, total, y) + vectors, spec, ptr(x),
              block.data_ptr(), at[0], at[1], ptr(gate), at[2], at[3], at[4], ptr(total), ptr(y))


def _tensor(t, name: str) -> None:
    if T.torch is None:
        T._bind()
    if not t.is_cuda:
        raise ValueError(f"{name} must be a cuda tensor")
    if t.dtype not in T._KINDS:
        raise ValueError(f"float32 or bfloat16 tensors, not {t.dtype}")
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
    if out is None:
        out = x.new_empty(x.shape)
    _call(None, x, True, weight, bias, gate, activation, None, None, None, eps, center, out, None, stream)
    return out


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
    T._require(x, "x", block.dtype, block.get_device(), block.shape)
    if weight is None and (bias is not None or out is not None):
        raise ValueError("bias and out come with weight")
    if block_weight is None and block_bias is not None:
        raise ValueError("block_bias comes with block_weight")
    if total is None:
        total = block.new_empty(block.shape)
    if out is None and weight is not None:
        out = block.new_empty(block.shape)
    if out is not None and block.numel() and out.data_ptr() == total.data_ptr():
        raise ValueError("total and out must be two tensors")
    _call(x, block, block_weight is not None, block_weight, block_bias, gate, activation, scale, weight, bias, eps, center,
          total, out, stream)
    return total, out
