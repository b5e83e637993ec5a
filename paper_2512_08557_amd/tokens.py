"""Token operators of libsscater.so: linear layers over rows of cells, and
attention over the tokens of earlier strides (argument marshalling only).

As in engine.py, tensors give device pointers and the HIP stream is torch's
current one unless another is passed; every value is computed in the library's
HIP kernels.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import numpy as np

from . import engine as E
from .engine import BF16, F32, _check, lib

ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "gelu": 2, "silu": 3}


def _kind(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise ValueError(f"float32 or bfloat16 tensors, not {t.dtype}")


def _require(t, name: str, like=None, dtype=None, shape=None):
    """A cuda tensor of the given dtype (or like's dtype and device) and shape."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a cuda tensor")
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")
    want = dtype if dtype is not None else like.dtype if like is not None else t.dtype
    if t.dtype != want:
        raise ValueError(f"{name} must be {want}, not {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, not {tuple(t.shape)}")
    return t


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr() if t is not None else None)


class _On:
    """The device of a call and its stream: a stream other than the current one
    first waits for it, and the call's tensors are recorded there."""

    def __init__(self, device, stream, tensors):
        import torch
        self._guard = torch.cuda.device(device)
        self._torch, self._stream, self._tensors = torch, stream, tensors

    def __enter__(self):
        self._guard.__enter__()
        cur = self._torch.cuda.current_stream()
        s = self._stream if self._stream is not None else cur
        if s != cur:
            s.wait_stream(cur)
            for t in self._tensors:
                if t is not None:
                    t.record_stream(s)
        return ctypes.c_void_p(s.cuda_stream)

    def __exit__(self, *exc):
        return self._guard.__exit__(*exc)


def _row_stride(t, name: str, width: int) -> int:
    """Elements between the rows of a tensor [..., width] whose leading axes
    run through one even stride."""
    if t.dim() < 1 or t.shape[-1] != width:
        raise ValueError(f"{name} must end in {width} values")
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
    import torch
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(k for k in ACTIVATIONS if k)}")
    kind = _kind(x)
    if weight.dim() != 2:
        raise ValueError("weight must be [cout, cin]")
    cout, cin = weight.shape
    _require(x, "x")
    _require(weight, "weight", like=x)
    shape = tuple(x.shape[:-1]) + (cout,)
    xs, ws = _row_stride(x, "x", cin), _row_stride(weight, "weight", cin)
    if bias is not None:
        _require(bias, "bias", like=x, shape=(cout,))
        if cout > 1 and bias.stride(0) != 1:
            raise ValueError("bias must be contiguous")
    rs = cout
    if residual is not None:
        rs = _row_stride(_require(residual, "residual", like=x, shape=shape), "residual", cout)
    if out is None:
        out = torch.empty(shape, dtype=x.dtype, device=x.device)
    ys = _row_stride(_require(out, "out", like=x, shape=shape), "out", cout)
    rows = out.numel() // cout
    spec = E.LinearSpec(rows, cin, cout, kind, ACTIVATIONS[activation], xs, ws, rs, ys)
    with _On(x.device, stream, (x, weight, bias, residual, out)) as s:
        _check(lib().sscater_linear(ctypes.byref(spec), _ptr(x), _ptr(weight), _ptr(bias), _ptr(residual), _ptr(out), s),
               "sscater_linear")
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
        import torch
        self.sections = tuple(int(n) for n in sections)
        if not 1 <= len(self.sections) <= 3 or any(n < 0 for n in self.sections):
            raise ValueError("one to three axes")
        if inv_freq is None:
            table = np.concatenate([base ** (-np.arange(n) / max(n, 1)) for n in self.sections])
            inv_freq = torch.from_numpy(table.astype(np.float32)).to(device)
        _require(inv_freq, "inv_freq", dtype=torch.float32, shape=(sum(self.sections),))
        if not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be contiguous")
        self.inv_freq = inv_freq
        self.interleaved = bool(interleaved)


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
        import torch
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
        for name, t in (("k", k), ("v", v)):
            _require(t, name, like=k, dtype=kind, shape=shape)
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
        self.k, self.v = k, v
        self.past = torch.zeros(self.batch, dtype=torch.int64, device=k.device)
        self.seen = 0

    def seek(self, past: Sequence[int]) -> None:
        """Streams that have seen past[b] tokens (0 for all: a new start)."""
        import torch
        past = [int(p) for p in past]
        if len(past) != self.batch or min(past) < 0:
            raise ValueError("one number of tokens per stream")
        self.past.copy_(torch.tensor(past, dtype=torch.int64))
        self.seen = max(past)

    def _spec(self):
        return E.TokenCacheSpec(F32 if self.dtype == "f32" else BF16, self.batch, self.kv_heads, self.head_dim,
                                self.sinks, self.capacity, self.k.data_ptr(), self.v.data_ptr(), self.past.data_ptr())

    def _rows(self, tokens: int, start, max_new: Optional[int]):
        import torch
        if start is None:
            if tokens % self.batch or (max_new is not None and max_new * self.batch != tokens):
                raise ValueError("without start every stream brings the same number of tokens")
            return E.TokenRows(tokens, tokens // self.batch, self.seen, None)
        _require(start, "start", like=self.past, dtype=torch.int32, shape=(self.batch + 1,))
        if not start.is_contiguous():
            raise ValueError("start must be contiguous")
        if max_new is None:
            max_new = tokens
        return E.TokenRows(tokens, max_new, self.seen, start.data_ptr())

    def append(self, qkv, pos, rotary: Rotary, q_heads: int, q_weight=None, k_weight=None, eps: float = 1e-6,
               start=None, max_new: Optional[int] = None, out=None, stream=None):
        """Projected rows qkv [tokens, (q_heads + 2 kv_heads) * head_dim] (query,
        key, value heads) into queries [tokens, q_heads, head_dim], returned, and
        keys and values, put into the cache at past[b] onwards.  Query and key
        heads are normalised (root mean square, q_weight and k_weight
        [head_dim]; None: not) and turned by pos (int32 [tokens, axes])."""
        import torch
        width = (q_heads + 2 * self.kv_heads) * self.head_dim
        _require(qkv, "qkv", like=self.k)
        if q_heads < 1 or qkv.dim() != 2:
            raise ValueError("qkv must be [tokens, (q_heads + 2 * kv_heads) * head_dim]")
        ld = _row_stride(qkv, "qkv", width)
        tokens = qkv.shape[0]
        if sum(rotary.sections) * 2 != self.head_dim:
            raise ValueError("the rotary sections must add up to head_dim / 2")
        _require(rotary.inv_freq, "inv_freq", like=self.past, dtype=torch.float32)
        _require(pos, "pos", like=self.past, dtype=torch.int32, shape=(tokens, len(rotary.sections)))
        if not pos.is_contiguous():
            raise ValueError("pos must be contiguous")
        if (q_weight is None) != (k_weight is None):
            raise ValueError("q_weight and k_weight come together")
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            if w is not None and not _require(w, name, like=self.k, shape=(self.head_dim,)).is_contiguous():
                raise ValueError(f"{name} must be contiguous")
        rows = self._rows(tokens, start, max_new)
        shape = (tokens, q_heads, self.head_dim)
        if out is None:
            out = torch.empty(shape, dtype=self.k.dtype, device=self.k.device)
        elif not _require(out, "out", like=self.k, shape=shape).is_contiguous():
            raise ValueError("out must be contiguous")
        section = (ctypes.c_int32 * 3)(*rotary.sections)
        spec = E.HeadSpec(q_heads, len(rotary.sections), section, int(rotary.interleaved), eps, ld)
        cache = self._spec()
        tensors = (qkv, pos, rotary.inv_freq, q_weight, k_weight, start, out, self.k, self.v, self.past)
        with _On(self.k.device, stream, tensors) as s:
            _check(lib().sscater_tokens_append(ctypes.byref(spec), ctypes.byref(cache), ctypes.byref(rows), _ptr(qkv),
                                               _ptr(q_weight), _ptr(k_weight), _ptr(rotary.inv_freq), _ptr(pos),
                                               _ptr(out), s), "sscater_tokens_append")
        return out

    def attend(self, q, window: int, start=None, max_new: Optional[int] = None, causal: bool = True,
               scale: Optional[float] = None, out=None, stream=None):
        """Attention of the call's queries q [tokens, q_heads, head_dim] (their
        keys and values appended, past not yet advanced) over the cache: a token
        sees the `window` newest tokens up to itself and the sinks (causal), or
        every new token of its stream and the window before them (not causal).
        scale: 1 / sqrt(head_dim) unless given."""
        import torch
        _require(q, "q", like=self.k)
        if q.dim() != 3 or q.shape[2] != self.head_dim or q.shape[1] < 1 or q.shape[1] % self.kv_heads:
            raise ValueError("q must be [tokens, q_heads, head_dim], q_heads a multiple of kv_heads")
        if not q.is_contiguous() or q.data_ptr() % 16:
            raise ValueError("q must be contiguous, on a 16-byte boundary")
        if window < 1:
            raise ValueError("window must be at least 1")
        rows = self._rows(q.shape[0], start, max_new)
        if out is None:
            out = torch.empty_like(q)
        elif not _require(out, "out", like=q, shape=q.shape).is_contiguous() or out.data_ptr() % 16:
            raise ValueError("out must be contiguous, on a 16-byte boundary")
        spec = E.AttendSpec(q.shape[1], min(int(window), 2 ** 31 - 1), int(bool(causal)),
                            self.head_dim ** -0.5 if scale is None else float(scale))
        cache = self._spec()
        need = ctypes.c_size_t()
        args = (ctypes.byref(spec), ctypes.byref(cache), ctypes.byref(rows))
        _check(lib().sscater_tokens_workspace(*args, ctypes.byref(need)), "sscater_tokens_workspace")
        work = torch.empty(need.value, dtype=torch.uint8, device=q.device) if need.value else None
        with _On(q.device, stream, (q, start, out, work, self.k, self.v, self.past)) as s:
            _check(lib().sscater_tokens_attend(*args, _ptr(q), _ptr(out), _ptr(work), need.value, s),
                   "sscater_tokens_attend")
        return out

    def advance(self, tokens: int, start=None, max_new: Optional[int] = None, stream=None) -> None:
        """The call's tokens become past ones."""
        rows = self._rows(int(tokens), start, max_new)
        cache = self._spec()
        with _On(self.past.device, stream, (start, self.past)) as s:
            _check(lib().sscater_tokens_advance(ctypes.byref(cache), ctypes.byref(rows), s), "sscater_tokens_advance")
        self.seen += rows.max_new
