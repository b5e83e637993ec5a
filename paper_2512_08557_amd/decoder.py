"""A decoder of object queries over a backbone's cells: norms, the delta memory and
cross attention as they run together, one call per stride.

A fixed number of queries lives through the strides.  In each, a query recalls and
corrects what it has seen (a DeltaMemory stream of its own), looks at the map's
occupied cells, and goes through a feed-forward layer; heads on the result are linear
calls.

    eng = Engine(...)                                  # the backbone
    dec = QueryDecoder(weights, queries=300, memory_heads=4, key_dim=32, value_dim=32,
                       q_heads=8, kv_heads=8, head_dim=32)
    x = query_embedding                                # [batch, 300, C]
    for ...:
        eng.step(idx, feats)
        cells = eng.read(16).view(1, -1, 256)
        x, y = dec.step(x, cells, mask=occupied)
        out = linear(y, w_head, b_head)
"""
from __future__ import annotations

from typing import Dict, Optional

from .cross import cross_attend
from .delta import DeltaMemory
from .norms import add_norm, norm
from .tokens import _require, _row_stride, _want_gradient, linear

NAMES = ("norm", "memory", "memory_gate", "memory_norm", "memory_out", "cross_norm", "q", "kv", "cross_out", "ffn_norm",
         "up", "down", "out_norm")
FLOATS = ("rate", "bias")
OPTIONAL = ("memory_scale", "cross_scale", "ffn_scale", "q_bias", "kv_bias", "cross_out_bias", "up_bias", "down_bias")


class QueryDecoder:
    """n = norm(x); x += s1 out1(silu(gate(n)) * norm(memory(n)));
    x += s2 out2(cross attention of norm(x) to the cells); x += s3 down(gelu(up(norm(x))));
    the result is x and norm(x).

    weights: cuda tensors of one dtype: the norms "norm", "cross_norm", "ffn_norm",
    "out_norm" [C] and "memory_norm" [value_dim]; "memory" [2 qk_heads * key_dim + heads *
    value_dim + 2 heads, C] (queries, keys, values, a, b), "memory_gate" [heads *
    value_dim, C], "memory_out" [C, heads * value_dim]; "q" [q_heads * head_dim, C], "kv"
    [2 kv_heads * head_dim, the cells' channels], "cross_out" [C, q_heads * head_dim];
    "up" [F, C], "down" [C, F]; biases "q_bias", "kv_bias", "cross_out_bias", "up_bias",
    "down_bias" and residual scales "memory_scale", "cross_scale", "ffn_scale" [C] where
    there are any; and, of float32, the memory's "rate" and "bias" [heads]."""

    def __init__(self, weights: Dict, queries: int, memory_heads: int, key_dim: int, value_dim: int, q_heads: int,
                 kv_heads: int, head_dim: int, qk_heads: Optional[int] = None, batch: int = 1, eps: float = 1e-6):
        import torch
        missing = [n for n in NAMES + FLOATS if n not in weights]
        if missing:
            raise ValueError(f"weights without {missing}")
        self.weights = {n: weights[n] for n in NAMES + FLOATS + OPTIONAL if weights.get(n) is not None}
        kind, index = weights["q"].dtype, weights["q"].get_device()
        dtype = {torch.float32: "f32", torch.bfloat16: "bf16"}.get(kind)
        if dtype is None:
            raise ValueError(f"weights must be float32 or bfloat16, not {kind}")
        other = [n for n in NAMES + OPTIONAL if weights.get(n) is not None and weights[n].dtype != kind]
        if other:
            raise ValueError(f"weights of one dtype: {other} differ from q")
        self.queries, self.batch, self.eps = int(queries), int(batch), eps
        self.q_heads, self.kv_heads, self.head_dim = int(q_heads), int(kv_heads), int(head_dim)
        self.memory = DeltaMemory(self.batch * self.queries, memory_heads, key_dim, value_dim, qk_heads=qk_heads,
                                  dtype=dtype, device=weights["q"].device)
        m = self.memory
        self.columns = [m.qk_heads * m.key_dim] * 2 + [m.heads * m.value_dim] + [m.heads] * 2
        # a weight that does not fit would be found in the middle of a stride, with the memory changed
        width, values, heads = weights["q"].shape[-1], m.heads * m.value_dim, self.q_heads * self.head_dim
        inner, cells = weights["up"].shape[0], weights["kv"].shape[-1]
        shapes = {"memory": (sum(self.columns), width), "memory_gate": (values, width), "memory_norm": (m.value_dim,),
                  "memory_out": (width, values), "q": (heads, width), "kv": (2 * self.kv_heads * self.head_dim, cells),
                  "cross_out": (width, heads), "up": (inner, width), "down": (width, inner), "q_bias": (heads,),
                  "kv_bias": (2 * self.kv_heads * self.head_dim,), "up_bias": (inner,), "rate": (m.heads,), "bias": (m.heads,)}
        for name in NAMES + FLOATS + OPTIONAL:
            if weights.get(name) is not None and tuple(weights[name].shape) != shapes.get(name, (width,)):
                raise ValueError(f"{name} must be {shapes.get(name, (width,))}, not {tuple(weights[name].shape)}")
        for name, t in self.weights.items():
            _require(t, name, torch.float32 if name in FLOATS else kind, index)
            if t.dim() == 1 and not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
            _row_stride(t, name, t.shape[-1])
        if self.kv_heads < 1 or self.q_heads % self.kv_heads or self.head_dim not in (32, 64, 128):
            raise ValueError("q_heads a multiple of kv_heads, head_dim 32, 64 or 128")

    def step(self, x, cells, mask=None):
        """One stride's queries x [batch, queries, C] and cells [batch, cells, channels],
        of which those with a true mask [batch, cells] are seen; x [batch, queries, C] for
        the next stride, and its norm."""
        import torch
        w, m, eps, width = self.weights, self.memory, self.eps, x.shape[-1]
        shape, n = (self.batch, self.queries, width), self.batch * self.queries
        # before the memory is changed, which a later refusal would leave so
        if x.requires_grad or any(t.requires_grad for t in w.values()):
            _want_gradient()
        if x.shape != shape:
            raise ValueError(f"x must be {shape}, not {tuple(x.shape)}")
        if cells.dim() != 3 or cells.shape[0] != self.batch or cells.shape[2] != w["kv"].shape[1]:
            raise ValueError(f"cells must be [{self.batch}, cells, {w['kv'].shape[1]}], not {tuple(cells.shape)}")
        if mask is not None and (mask.dtype not in (torch.bool, torch.uint8) or mask.shape != cells.shape[:2] or
                                 mask.device != x.device or not mask.is_contiguous()):
            raise ValueError(f"mask must be a contiguous bool or uint8 tensor {tuple(cells.shape[:2])} on {x.device}")
        kv = linear(cells, w["kv"], w.get("kv_bias")).view(self.batch, -1, 2, self.kv_heads, self.head_dim)
        x = x.reshape(n, width)
        h = norm(x, w["norm"], eps=eps)
        q, k, v, a, b = linear(h, w["memory"]).split(self.columns, 1)
        o = m.update(q.unflatten(1, (m.qk_heads, m.key_dim)), k.unflatten(1, (m.qk_heads, m.key_dim)),
                     v.unflatten(1, (m.heads, m.value_dim)), a, b, rate=w["rate"], bias=w["bias"], eps=eps)
        gate = linear(h, w["memory_gate"]).view(o.shape)
        o = norm(o, w["memory_norm"], eps=eps, gate=gate, activation="silu", out=o)
        y = linear(o.view(n, -1), w["memory_out"])
        x, h = add_norm(x, y, w["cross_norm"], scale=w.get("memory_scale"), eps=eps)
        q = linear(h, w["q"], w.get("q_bias")).view(self.batch, self.queries, self.q_heads, self.head_dim)
        c = cross_attend(q, kv[:, :, 0], kv[:, :, 1], mask)
        y = linear(c.view(n, -1), w["cross_out"], w.get("cross_out_bias"))
        x, h = add_norm(x, y, w["ffn_norm"], scale=w.get("cross_scale"), eps=eps, total=x)
        y = linear(linear(h, w["up"], w.get("up_bias"), activation="gelu"), w["down"], w.get("down_bias"))
        x, h = add_norm(x, y, w["out_norm"], scale=w.get("ffn_scale"), eps=eps, total=x)
        return x.view(shape), h.view(shape)

    def reset(self) -> None:
        """Forget every stride."""
        self.memory.reset()
