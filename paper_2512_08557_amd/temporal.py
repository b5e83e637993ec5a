"""A temporal block over the cells of a backbone's map: the token operators as
they run together, one call per stride.

Each cell of a coarse map is a token.  A stride's tokens attend to one another,
to those of the last strides (a sliding window in a TokenCache) and to the first
tokens the sensor ever gave, and go through a feed-forward layer; a 1x1 head on
the result is one more linear call.

    eng = Engine(...)                                  # the backbone
    block = TemporalBlock(weights, q_heads=8, kv_heads=8, head_dim=32, tokens=62 * 54, strides=10)
    head = lambda y: linear(y, w_head, b_head)
    for ...:
        eng.step(idx, feats)
        y = block.step(eng.read(16).view(-1, 256), stride, (62, 54))
        out = head(y)
"""
from __future__ import annotations

from typing import Dict, Optional, Sequence, Tuple

from .tokens import Rotary, TokenCache, linear

NAMES = ("qkv", "q_norm", "k_norm", "out", "up", "down")
BIASES = ("qkv_bias", "out_bias", "up_bias", "down_bias")


class TemporalBlock:
    """y = x + out(attention(x)), z = y + down(gelu(up(y))).

    weights: cuda tensors of one dtype: "qkv" [(q_heads + 2 kv_heads) * head_dim,
    C], "q_norm" and "k_norm" [head_dim], "out" [C, q_heads * head_dim], "up"
    [F, C], "down" [C, F], and biases "qkv_bias", "out_bias", "up_bias",
    "down_bias" where there are any.  tokens: the most a stride brings; strides:
    how many of them before the present one are looked back over; sinks: first
    tokens that stay.  sections: pairs of a head that turn with the stride, the
    row and the column (a half, a quarter and a quarter unless given)."""

    def __init__(self, weights: Dict, q_heads: int, kv_heads: int, head_dim: int, tokens: int, strides: int,
                 sinks: int = 16, sections: Optional[Sequence[int]] = None, batch: int = 1):
        import torch
        missing = [n for n in NAMES if n not in weights]
        if missing:
            raise ValueError(f"weights without {missing}")
        self.weights = dict(weights)
        self.q_heads, self.batch = int(q_heads), int(batch)
        # a stride's tokens and the ones before them
        self.window, self.tokens = strides * tokens + 1, int(tokens)
        dtype = {torch.float32: "f32", torch.bfloat16: "bf16"}.get(weights["qkv"].dtype)
        if dtype is None:
            raise ValueError(f"weights must be float32 or bfloat16, not {weights['qkv'].dtype}")
        other = [n for n in NAMES + BIASES if weights.get(n) is not None and weights[n].dtype != weights["qkv"].dtype]
        if other:
            raise ValueError(f"weights of one dtype: {other} differ from qkv")
        device = weights["qkv"].device
        self.cache = TokenCache(batch, kv_heads, head_dim, sinks + self.window + tokens - 1, sinks=sinks, dtype=dtype,
                                device=device)
        self.rotary = Rotary(None, sections or (head_dim // 4, head_dim // 8, head_dim // 8), device=device)
        self._grid: Optional[Tuple] = None
        self._pos = None

    def positions(self, stride: int, grid: Tuple[int, int]):
        """(stride, row, column) of every cell of `batch` maps, int32 [batch * H * W, 3]."""
        import torch
        if self._grid != tuple(grid):
            h, w = grid
            pos = torch.empty(self.batch, h, w, 3, dtype=torch.int32, device=self.cache.k.device)
            pos[..., 1] = torch.arange(h, dtype=torch.int32, device=pos.device)[:, None]
            pos[..., 2] = torch.arange(w, dtype=torch.int32, device=pos.device)
            self._grid, self._pos = tuple(grid), pos.view(-1, 3)
        self._pos[:, 0] = stride
        return self._pos

    def step(self, x, stride: int, grid: Tuple[int, int]):
        """One stride's cells x [batch * H * W, C], at most `tokens` of a map; the
        result has their shape."""
        w, n = self.weights, x.shape[0]
        # before anything is put into the cache, where more of them would go over tokens that are still looked back at
        if grid[0] * grid[1] > self.tokens:
            raise ValueError(f"a map of {grid[0]} x {grid[1]} cells: a stride brings at most {self.tokens}")
        qkv = linear(x, w["qkv"], w.get("qkv_bias"))
        q = self.cache.append(qkv, self.positions(stride, grid), self.rotary, self.q_heads, q_weight=w["q_norm"],
                              k_weight=w["k_norm"])
        a = self.cache.attend(q, self.window, causal=False)
        self.cache.advance(n)
        y = linear(a.view(n, -1), w["out"], w.get("out_bias"), residual=x)
        h = linear(y, w["up"], w.get("up_bias"), activation="gelu")
        return linear(h, w["down"], w.get("down_bias"), residual=y)

    def reset(self) -> None:
        """Forget every stride."""
        self.cache.seek([0] * self.batch)
