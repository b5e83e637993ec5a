"""Token operators of libsscater.so: linear layers over rows of cells, and
attention over the tokens of earlier strides (argument marshalling only).  They
form no gradients: where one would be wanted they refuse the call.

As in engine.py, tensors give device pointers and the HIP stream is torch's
current one unless another is passed; every value is computed in the library's
HIP kernels.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import numpy as np

from . import engine as E
from .engine import BF16, F32, SscaterError, _check, lib

ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "gelu": 2, "silu": 3}


torch = _device = _stream = None
_KINDS: dict = {}


def _bind():
    """torch, at the first call (as in Engine), and its current device and
    stream as plain numbers: the objects around them cost more than a launch.
    torch comes last: callers on other threads take it for a sign of the rest."""
    global torch, _device, _stream
    import torch as t
    _KINDS.update({t.float32: F32, t.bfloat16: BF16})
    _device, _stream = t._C._cuda_getDevice, t._C._cuda_getCurrentRawStream
    torch = t


def _require(t, name: str, dtype, index: int, shape=None):
    """A cuda tensor of the given dtype on device `index`, of the given shape."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a cuda tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{index}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, not {tuple(t.shape)}")
    return t


def _dense(t, name: str, dtype, index: int, shape):
    if not _require(t, name, dtype, index, shape).is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _want_gradient() -> None:
    """Called for operands that require a gradient: a result without one would be
    taken for a constant; and for tensors that are written and require one: what
    autograd holds of them would not know of it."""
    if torch.is_grad_enabled():
        raise ValueError("no gradient is formed: detach the operands or call under torch.no_grad()")


def _number(value) -> float:
    """A scale or an eps as a plain number: of a tensor what it holds now (descriptions of
    calls are kept by their values, and a tensor is found by what it is, not holds)."""
    if type(value) is float:
        return value
    if getattr(value, "requires_grad", False):
        _want_gradient()
    return float(value)


def _launch(fn, where: str, index: int, stream, tensors, *args) -> None:
    """One library call on device `index`, on torch's current stream; another
    stream first waits for that one, and the call's tensors are recorded there
    (as in Engine)."""
    if stream is None and _device() == index:
        rc = fn(*args, _stream(index))
    else:
        with torch.cuda.device(index):
            cur = torch.cuda.current_stream()
            s = stream if stream is not None else cur
            if s != cur:
                s.wait_stream(cur)
                for t in tensors:
                    if t is not None:
                        t.record_stream(s)
            rc = fn(*args, s.cuda_stream)
    if rc != E.OK:
        raise SscaterError(rc, where)


def _row_stride(t, name: str, width: int) -> int:
    """Elements between the rows of a tensor [..., width] whose leading axes
    run through one even stride."""
    if t.dim() < 1 or t.shape[-1] != width:
        raise ValueError(f"{name} must end in {width} values")
    if t.is_contiguous():
        return width
    if width > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the values of a row must be contiguous")
    if t.numel() == 0:
        return width
    step, n = None, 1
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if step is None:
            step = stride
        elif stride != step * n:
            raise ValueError(f"{name}: its rows must lie evenly apart")
        n *= size
    if step is None:
        return width
    if step < width:
        raise ValueError(f"{name}: its rows overlap")
    return step


def linear(x, weight, bias=None, activation: Optional[str] = None, residual=None, out=None, stream=None):
    """act(x W^T + bias) + residual.  x [..., cin] (float32 or bfloat16, its
    rows evenly apart), weight [cout, cin], bias [cout], residual and out
    [..., cout]; activation none, relu, gelu or silu.  out may be the residual
    and must not overlap the other operands."""
    act = ACTIVATIONS.get(activation, -1)
    if act < 0:
        raise ValueError(f"activation must be one of {sorted(k for k in ACTIVATIONS if k)}")
    if torch is None:
        _bind()
    dtype = x.dtype
    kind = _KINDS.get(dtype, -1)
    if kind < 0:
        raise ValueError(f"float32 or bfloat16 tensors, not {dtype}")
    if weight.dim() != 2 or 0 in weight.shape:
        raise ValueError("weight must be [cout, cin], of at least one channel each")
    cout, cin = weight.shape
    if not x.is_cuda:
        raise ValueError("x must be a cuda tensor")
    index = x.get_device()
    _require(weight, "weight", dtype, index)
    xs, ws, rs = _row_stride(x, "x", cin), _row_stride(weight, "weight", cin), cout
    shape = x.shape[:-1] + (cout,)
    if bias is not None:
        _require(bias, "bias", dtype, index, (cout,))
        if cout > 1 and bias.stride(0) != 1:
            raise ValueError("bias must be contiguous")
    if residual is not None:
        rs = _row_stride(_require(residual, "residual", dtype, index, shape), "residual", cout)
    if x.requires_grad or weight.requires_grad or (bias is not None and bias.requires_grad) or \
            (residual is not None and residual.requires_grad):
        _want_gradient()
    if out is None:
        out, ys = x.new_empty(shape), cout
    else:
        ys = _row_stride(_require(out, "out", dtype, index, shape), "out", cout)
        if out.requires_grad:
            _want_gradient()
    spec = E.LinearSpec(x.numel() // cin, cin, cout, kind, act, xs, ws, rs, ys)
    _launch(lib().sscater_linear, "sscater_linear", index, stream, (x, weight, bias, residual, out), spec, x.data_ptr(),
            weight.data_ptr(), None if bias is None else bias.data_ptr(),
            None if residual is None else residual.data_ptr(), out.data_ptr())
    return out


class Rotary:
    """Rotary positions with one to three axes (stride, row, column): the
    head_dim / 2 pairs of a head are turned by position * inv_freq, the first
    sections[0] pairs by the first axis's position, and so on.  inv_freq: float32
    cuda tensor [head_dim / 2], or None for base ** (-i / sections[a]) within
    each axis's pairs.  interleaved: a pair is two neighbouring values instead of
    one of either half of the head."""

    def __init__(self, inv_freq, sections: Sequence[int], interleaved: bool = False, base: float = 10000.0,
                 device="cuda"):
        if torch is None:
            _bind()
        self.sections = tuple(int(n) for n in sections)
        if not 1 <= len(self.sections) <= 3 or any(n < 0 for n in self.sections):
            raise ValueError("one to three axes")
        if inv_freq is None:
            table = np.concatenate([base ** (-np.arange(n) / max(n, 1)) for n in self.sections])
            inv_freq = torch.from_numpy(table.astype(np.float32)).to(device)
        _dense(inv_freq, "inv_freq", torch.float32, inv_freq.get_device(), (sum(self.sections),))
        self.inv_freq = inv_freq
        self.interleaved = int(bool(interleaved))
        self.section = (ctypes.c_int32 * 3)(*self.sections)


class TokenCache:
    """Keys and values of the tokens of `batch` streams, for attention that
    looks back over a sliding window and the first `sinks` tokens.  Token j of a
    stream sits in slot j if j < sinks, else in slot sinks + (j - sinks) %
    (capacity - sinks); k and v are [batch, kv_heads, capacity, head_dim] tensors
    (zeros, or the caller's), past counts the tokens that each stream has seen.

    A call's new tokens are rows of one tensor: sequence b's are rows start[b]
    to start[b + 1] - 1 (start: int32 cuda tensor [batch + 1], max_new the most
    rows of one sequence), or, without start, the same number for each.  Per
    stride: append, attend, advance.  Calls replayed from a graph do not move
    the host's bound on past (`seen`): capture with the capacity of the whole
    reach, sinks + window + max_new - 1, which needs no bound."""

    def __init__(self, batch: int, kv_heads: int, head_dim: int, capacity: int, sinks: int = 0, dtype: str = "f32",
                 k=None, v=None, device="cuda"):
        if torch is None:
            _bind()
        if dtype not in ("f32", "bf16"):
            raise ValueError("dtype must be f32 or bf16")
        if batch < 1 or kv_heads < 1 or head_dim not in (32, 64, 128):
            raise ValueError("batch and kv_heads of at least 1, head_dim 32, 64 or 128")
        if sinks < 0 or capacity <= sinks:
            raise ValueError("capacity must exceed sinks")
        self.batch, self.kv_heads, self.head_dim = int(batch), int(kv_heads), int(head_dim)
        self.capacity, self.sinks, self.dtype = int(capacity), int(sinks), dtype
        kind = torch.float32 if dtype == "f32" else torch.bfloat16
        shape = (self.batch, self.kv_heads, self.capacity, self.head_dim)
        if (k is None) != (v is None):
            raise ValueError("k and v come together")
        if k is None:
            k, v = (torch.zeros(shape, dtype=kind, device=device) for _ in range(2))
        self.index = k.get_device()
        for name, t in (("k", k), ("v", v)):
            _dense(t, name, kind, self.index, shape)
        self._k, self._v, self.kind = k, v, kind
        self._past = torch.zeros(self.batch, dtype=torch.int64, device=k.device)
        self.seen = 0
        self._spec = E.TokenCacheSpec(F32 if dtype == "f32" else BF16, self.batch, self.kv_heads, self.head_dim,
                                      self.sinks, self.capacity, k.data_ptr(), v.data_ptr(), self._past.data_ptr())

    # the library's description of the cache holds their addresses: they are filled, not replaced
    k = property(lambda self: self._k)
    v = property(lambda self: self._v)
    past = property(lambda self: self._past)

    def seek(self, past: Sequence[int]) -> None:
        """Streams that have seen past[b] tokens (0 for all: a new start)."""
        past = [int(p) for p in past]
        if len(past) != self.batch or min(past) < 0:
            raise ValueError("one number of tokens per stream")
        if min(past) == max(past):
            self._past.fill_(past[0])
        else:
            self._past.copy_(torch.tensor(past, dtype=torch.int64))
        self.seen = max(past)

    def _rows(self, tokens: int, start, max_new: Optional[int]):
        if start is None:
            if tokens % self.batch or (max_new is not None and max_new * self.batch != tokens):
                raise ValueError("without start every stream brings the same number of tokens")
            return E.TokenRows(tokens, tokens // self.batch, self.seen, None)
        ptr = _dense(start, "start", torch.int32, self.index, (self.batch + 1,))
        return E.TokenRows(tokens, tokens if max_new is None else max_new, self.seen, ptr)

    def append(self, qkv, pos, rotary: Rotary, q_heads: int, q_weight=None, k_weight=None, eps: float = 1e-6,
               start=None, max_new: Optional[int] = None, out=None, stream=None):
        """Projected rows qkv [tokens, (q_heads + 2 kv_heads) * head_dim] (query,
        key, value heads) into queries [tokens, q_heads, head_dim], returned, and
        keys and values, put into the cache at past[b] onwards.  Query and key
        heads are normalised (root mean square, q_weight and k_weight
        [head_dim]; None: not) and turned by pos (int32 [tokens, axes])."""
        index, dim = self.index, self.head_dim
        _require(qkv, "qkv", self.kind, index)
        if q_heads < 1 or qkv.dim() != 2:
            raise ValueError("qkv must be [tokens, (q_heads + 2 * kv_heads) * head_dim]")
        ld = _row_stride(qkv, "qkv", (q_heads + 2 * self.kv_heads) * dim)
        tokens, axes = qkv.shape[0], len(rotary.sections)
        freq = _dense(rotary.inv_freq, "inv_freq: head_dim / 2 values,", torch.float32, index, (dim // 2,))
        at = _dense(pos, "pos", torch.int32, index, (tokens, axes))
        if (q_weight is None) != (k_weight is None):
            raise ValueError("q_weight and k_weight come together")
        qw = kw = None
        if q_weight is not None:
            qw, kw = (_dense(w, "q_weight and k_weight", self.kind, index, (dim,)) for w in (q_weight, k_weight))
            if q_weight.requires_grad or k_weight.requires_grad:
                _want_gradient()
        if qkv.requires_grad or self._k.requires_grad or self._v.requires_grad:
            _want_gradient()
        rows = self._rows(tokens, start, max_new)
        shape = (tokens, q_heads, dim)
        if out is None:
            out = qkv.new_empty(shape)
        else:
            _dense(out, "out", self.kind, index, shape)
            if out.requires_grad:
                _want_gradient()
        spec = E.HeadSpec(q_heads, axes, rotary.section, rotary.interleaved, _number(eps), ld)
        _launch(lib().sscater_tokens_append, "sscater_tokens_append", index, stream,
                (qkv, pos, rotary.inv_freq, q_weight, k_weight, start, out, self.k, self.v, self.past), spec,
                self._spec, rows, qkv.data_ptr(), qw, kw, freq, at, out.data_ptr())
        return out

    def attend(self, q, window: int, start=None, max_new: Optional[int] = None, causal: bool = True,
               scale: Optional[float] = None, out=None, stream=None):
        """Attention of the call's queries q [tokens, q_heads, head_dim] (their
        keys and values appended, past not yet advanced) over the cache: a token
        sees the `window` newest tokens up to itself and the sinks (causal), or
        every new token of its stream and the window before them (not causal).
        scale: 1 / sqrt(head_dim) unless given.  bfloat16: where a stream may
        bring more than 32 rows (max_new * q_heads / kv_heads) probabilities are
        rounded to bfloat16 for the product with the values."""
        index = self.index
        _require(q, "q", self.kind, index)
        if q.dim() != 3 or q.shape[2] != self.head_dim or q.shape[1] < 1 or q.shape[1] % self.kv_heads:
            raise ValueError("q must be [tokens, q_heads, head_dim], q_heads a multiple of kv_heads")
        if not q.is_contiguous() or q.data_ptr() % 16:
            raise ValueError("q must be contiguous, on a 16-byte boundary")
        if window < 1:
            raise ValueError("window must be at least 1")
        if q.requires_grad or self._k.requires_grad or self._v.requires_grad:
            _want_gradient()
        rows = self._rows(q.shape[0], start, max_new)
        if out is None:
            out = q.new_empty(q.shape)
        elif _dense(out, "out", self.kind, index, q.shape) % 16:
            raise ValueError("out must be on a 16-byte boundary")
        elif out.requires_grad:
            _want_gradient()
        spec = E.AttendSpec(q.shape[1], min(int(window), 2 ** 31 - 1), 1 if causal else 0,
                            self.head_dim ** -0.5 if scale is None else _number(scale))
        cache, need, work = self._spec, ctypes.c_size_t(), None
        _check(lib().sscater_tokens_workspace(spec, cache, rows, need), "sscater_tokens_workspace")
        if need.value:
            work = q.new_empty(need.value, dtype=torch.uint8)
        _launch(lib().sscater_tokens_attend, "sscater_tokens_attend", index, stream,
                (q, start, out, work, self.k, self.v, self.past), spec, cache, rows, q.data_ptr(), out.data_ptr(),
                None if work is None else work.data_ptr(), need.value)
        return out

    def advance(self, tokens: int, start=None, max_new: Optional[int] = None, stream=None) -> None:
        """The call's tokens become past ones."""
        rows = self._rows(int(tokens), start, max_new)
        _launch(lib().sscater_tokens_advance, "sscater_tokens_advance", self.index, stream, (start, self.past),
                self._spec, rows)
        self.seen += rows.max_new
