"""The gated delta rule of libsscater.so (argument marshalling only).  It forms no
gradients: where one would be wanted it refuses the call."""
from __future__ import annotations

import ctypes
from typing import Optional

from . import engine as E
from . import tokens as T
from .engine import BF16, F32, _check, lib


class DeltaMemory:
    """What `batch` streams of tokens remember, at a size that does not grow with
    them: for each of `heads` value heads a matrix S [key_dim, value_dim] (state,
    float32 [batch, heads, key_dim, value_dim]; zeros, or the caller's), which every
    token corrects and reads:

        u = beta (v - alpha S^T k),  S <- alpha S + k u^T,  out = scale S^T q

    Value head h takes query and key head h / (heads / qk_heads).  key_dim and
    value_dim 32, 64 or 128."""

    def __init__(self, batch: int, heads: int, key_dim: int, value_dim: int, qk_heads: Optional[int] = None,
                 dtype: str = "f32", state=None, device="cuda"):
        if T.torch is None:
            T._bind()
        torch = T.torch
        if dtype not in ("f32", "bf16"):
            raise ValueError("dtype must be f32 or bf16")
        qk_heads = heads if qk_heads is None else qk_heads
        if batch < 1 or heads < 1 or qk_heads < 1 or heads % qk_heads:
            raise ValueError("batch and heads of at least 1, heads a multiple of qk_heads")
        if key_dim not in (32, 64, 128) or value_dim not in (32, 64, 128):
            raise ValueError("key_dim and value_dim 32, 64 or 128")
        self.batch, self.heads, self.qk_heads = int(batch), int(heads), int(qk_heads)
        self.key_dim, self.value_dim, self.dtype = int(key_dim), int(value_dim), dtype
        shape = (self.batch, self.heads, self.key_dim, self.value_dim)
        if state is None:
            state = torch.zeros(shape, dtype=torch.float32, device=device)
        self.index = state.get_device()
        if T._dense(state, "state", torch.float32, self.index, shape) % 16:
            raise ValueError("state must be on a 16-byte boundary")
        self._state, self.kind = state, torch.float32 if dtype == "f32" else torch.bfloat16
        self._spec = E.DeltaMemorySpec(F32 if dtype == "f32" else BF16, self.batch, self.heads, self.qk_heads,
                                       self.key_dim, self.value_dim, state.data_ptr())

    # the library's description of the memory holds its address: it is filled, not replaced
    state = property(lambda self: self._state)

    def reset(self) -> None:
        """Forget everything."""
        self._state.zero_()

    def _row(self, t, name: str, tokens: int, heads: int, dim: int) -> int:
        """The stride from token to token of [tokens, heads, dim] (dim 0: [tokens,
        heads]), a token's values contiguous."""
        shape, stride = t.shape, t.stride()
        if t.dtype is not self.kind or t.get_device() != self.index or len(shape) != (3 if dim else 2) or \
                shape[0] != tokens or shape[1] != heads or (dim and shape[2] != dim):
            T._require(t, name, self.kind, self.index, (tokens, heads, dim) if dim else (tokens, heads))
        if t.requires_grad:
            T._want_gradient()
        if dim and stride[2] != 1 or heads > 1 and stride[1] != (dim or 1):
            raise ValueError(f"{name}: a token's values must be contiguous")
        width = heads * (dim or 1)
        if tokens < 2:
            return width
        if stride[0] < width:
            raise ValueError(f"{name}: its tokens overlap")
        return stride[0]

    def update(self, q, k, v, a, b, rate=None, bias=None, eps: Optional[float] = 1e-6, scale: Optional[float] = None,
               start=None, max_new: Optional[int] = None, initial=None, out=None, stream=None):
        """The new tokens of every stream, one after the other; what they read,
        [tokens, heads, value_dim], is returned.

        q and k [tokens, qk_heads, key_dim], v [tokens, heads, value_dim], a and b
        [tokens, heads], all of the memory's dtype; each may be columns of a
        projection's rows.  A call's tokens are rows as for TokenCache: sequence b's are
        start[b] to start[b + 1] - 1 (start: int32 cuda tensor [batch + 1], max_new the
        most of one stream), or, without start, the same number for each.  Queries and
        keys are taken to unit length, x / sqrt(sum x^2 + eps) (eps None: not).  rate
        and bias (float32 [heads]): alpha = exp(-rate softplus(a + bias)) and beta =
        sigmoid(b); without them alpha = exp(a), a <= 0, and beta = b.  scale: 1 /
        sqrt(key_dim) unless given.  initial: states to begin from instead of the
        memory's (which are written all the same).  out: the result's shape, contiguous;
        it and the state overlap no operand (initial may be the state itself).  Long
        streams take a workspace of 21.6 KB for every 64 tokens and head."""
        index = self.index
        if self._state.requires_grad:
            T._want_gradient()
        if q.dim() != 3:
            raise ValueError("q must be [tokens, qk_heads, key_dim]")
        tokens = q.shape[0]
        if start is None:
            if tokens % self.batch or (max_new is not None and max_new * self.batch != tokens):
                raise ValueError("without start every stream brings the same number of tokens")
            rows = E.TokenRows(tokens, tokens // self.batch, 0, None)
        else:
            rows = E.TokenRows(tokens, tokens if max_new is None else max_new, 0,
                               T._dense(start, "start", T.torch.int32, index, (self.batch + 1,)))
        heads = self.heads
        ldq, ldk = self._row(q, "q", tokens, self.qk_heads, self.key_dim), self._row(k, "k", tokens, self.qk_heads, self.key_dim)
        ldv = self._row(v, "v", tokens, heads, self.value_dim)
        lda, ldb = self._row(a, "a", tokens, heads, 0), self._row(b, "b", tokens, heads, 0)
        if (rate is None) != (bias is None):
            raise ValueError("rate and bias come together")
        if rate is not None:
            for name, t in (("rate", rate), ("bias", bias)):
                T._dense(t, name, T.torch.float32, index, (heads,))
                if t.requires_grad:
                    T._want_gradient()
        if initial is not None:
            if T._dense(initial, "initial", T.torch.float32, index, self._state.shape) % 16:
                raise ValueError("initial must be on a 16-byte boundary")
            if initial.requires_grad:
                T._want_gradient()
        shape = (tokens, heads, self.value_dim)
        if out is None:
            out = q.new_empty(shape)
        elif T._dense(out, "out", self.kind, index, shape) % 16:
            raise ValueError("out must be on a 16-byte boundary")
        elif out.requires_grad:
            T._want_gradient()
        spec = E.DeltaSpec(0 if eps is None else 1, 0.0 if eps is None else T._number(eps),
                           self.key_dim ** -0.5 if scale is None else T._number(scale), ldq, ldk, ldv, lda, ldb)
        need, work = ctypes.c_size_t(), None
        _check(lib().sscater_delta_workspace(spec, self._spec, rows, need), "sscater_delta_workspace")
        if need.value:
            work = q.new_empty(need.value, dtype=T.torch.uint8)
        T._launch(lib().sscater_delta_update, "sscater_delta_update", index, stream,
                  (q, k, v, a, b, rate, bias, initial, start, out, work, self._state), spec, self._spec, rows,
                  None if initial is None else initial.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), a.data_ptr(),
                  b.data_ptr(), None if rate is None else rate.data_ptr(), None if bias is None else bias.data_ptr(),
                  out.data_ptr(), None if work is None else work.data_ptr(), need.value)
        return out
