"""Timed cases of the operators behind a decoder of object queries over the maps' cells.

  norm    the norms around a block: s = x + scale * act(gate) * P(block) and y = N(s) (add_norm), or
          y = act(gate) * N(x) (norm)
  cross   attention of one set of tokens to another: object queries to a map's cells, of which only the
          occupied ones may be visible
  delta   the gated delta rule: a memory of fixed size for every stream and head, token by token or over
          whole stretches of a stream

A case's fields:
  op      norm | cross | delta
  dtype   f32 | bf16
 norm:
  rows, width
  block   whether there are a block's output and a residual stream (add_norm) or only x (norm)
  center  whether the mean is taken off
  post    whether the block's output is normalised before it is added
  bias    whether the norms have one
  gate    none | row (a row of its own for every row) | image (one for each of `images` runs of rows)
  act     of the gate: none | sigmoid | silu
  scale   whether the block's output is scaled channel by channel
 cross:
  batch, queries, keys   sequences, and the most queries and keys of one of them
  ragged  whether the sequences have different numbers of both (otherwise they are one dense tensor)
  visible share of the keys that can be seen (1: no mask)
  q_heads, kv_heads, dim
  fused   whether keys and values are columns of one projection's rows
 delta:
  batch, new   streams, and the new tokens of the longest of them
  ragged  whether the streams bring different numbers of tokens
  heads, qk_heads, key_dim, value_dim
"""
import math
import random

import numpy as np
import torch

own = False            # the library's operators (True), or their plain forms in torch

MAP = 248 * 216        # cells of the first block's and the neck's map
COARSE = 62 * 54       # cells of the last block's map
EPS = 1e-6
CHUNK = 64


def _norm(dtype, rows, width, block=True, center=False, post=False, bias=False, gate="none", act="none", scale=False,
          images=1, **more):
    return dict(op="norm", dtype=dtype, rows=rows, width=width, block=block, center=center, post=post, bias=bias,
                gate=gate, act=act, scale=scale, images=images, **more)


def _cross(dtype, batch, queries, keys, q_heads, kv_heads, dim, visible=1.0, ragged=False, fused=True, **more):
    return dict(op="cross", dtype=dtype, batch=batch, queries=queries, keys=keys, q_heads=q_heads, kv_heads=kv_heads,
                dim=dim, visible=visible, ragged=ragged, fused=fused, **more)


def _delta(dtype, batch, new, heads, key_dim, value_dim, qk_heads=0, ragged=False, **more):
    return dict(op="delta", dtype=dtype, batch=batch, new=new, heads=heads, qk_heads=qk_heads or heads,
                key_dim=key_dim, value_dim=value_dim, ragged=ragged, **more)


def listed():
    return [
        # four sensors' one token each after a block: launch and latency
        _norm("bf16", 4, 256, post=True, name="norm_token_bf16"),
        # the heads of a memory over a coarse map's cells, each normalised and gated by a projection of its own
        _norm("f32", 8 * COARSE, 32, block=False, gate="row", act="silu", name="norm_heads_f32"),
        # four sensors' neck maps after a block: normalised, gated by each image's condition, scaled, added and
        # normalised for the next one
        _norm("bf16", 4 * MAP, 384, center=True, post=True, bias=True, gate="image", images=4, act="sigmoid", scale=True,
              name="norm_map_bf16"),
        # one query of each of four sensors over its coarse map: launch and latency
        _cross("bf16", 4, 1, COARSE, 8, 8, 32, name="cross_token_bf16"),
        # object queries over a coarse map
        _cross("f32", 1, 300, COARSE, 8, 8, 32, name="cross_objects_f32"),
        # the object queries of four sensors over the occupied cells of their first maps
        _cross("bf16", 4, 900, MAP, 8, 8, 32, visible=0.224, name="cross_occupied_bf16"),
        # sequences of different lengths, one of them without a visible cell
        _cross("f32", 9, 257, 12001, 4, 1, 128, visible=0.6, ragged=True, fused=False, name="cross_ragged_f32"),
        # the object queries of four sensors over every cell of their neck maps
        _cross("bf16", 4, 900, MAP, 16, 4, 64, name="cross_map_bf16"),
        # one token of each of four streams: launch and latency
        _delta("bf16", 4, 1, 8, 64, 64, name="delta_token_bf16"),
        # every cell of a coarse map its own stream, one token a stride
        _delta("f32", COARSE, 1, 8, 32, 32, name="delta_cells_f32"),
        # a stride's cells one after the other through one memory
        _delta("bf16", 1, COARSE, 8, 64, 64, name="delta_stride_bf16"),
        # whole windows of four streams, of different lengths, two value heads for each key head
        _delta("f32", 4, 10 * COARSE, 8, 64, 128, qk_heads=4, ragged=True, name="delta_window_f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    flops = 1e15 if case["dtype"] == "bf16" and case["op"] == "cross" else 1e14
    return max(w["flops"] / flops, w["bytes"] / 4e12)


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("norm", "cross", "delta")}
    op = rng.choice(sorted(most))
    while True:
        dtype = rng.choice(["f32", "bf16"])
        if op == "norm":
            gate = rng.choice(["none", "row", "image"])
            images = _log_int(rng, 1, 16) if gate == "image" else 1
            case = _norm(dtype, _log_int(rng, 1, 8 * COARSE * 8), _log_int(rng, 8, 2048), block=rng.random() < 0.7,
                         center=rng.random() < 0.4, post=rng.random() < 0.5, bias=rng.random() < 0.4, gate=gate,
                         act=rng.choice(["none", "sigmoid", "silu"]) if gate != "none" else "none",
                         scale=rng.random() < 0.4, images=images)
            case["rows"] = -(-case["rows"] // images) * images
            if rng.random() < 0.7:      # most widths are multiples of 16
                case["width"] = -(-case["width"] // 16) * 16
        elif op == "cross":
            kv = rng.choice([1, 2, 4, 8])
            case = _cross(dtype, _log_int(rng, 1, 16), rng.choice([1, 1, 2, 7, _log_int(rng, 8, 1000), _log_int(rng, 8, 1000)]),
                          _log_int(rng, 1, MAP), kv * rng.choice([1, 1, 2, 4]), kv, rng.choice([32, 64, 128]),
                          visible=rng.choice([1.0, 1.0, 0.6, 0.25, 0.05]), ragged=rng.random() < 0.4,
                          fused=rng.random() < 0.6)
        else:
            form = rng.choice(["cells", "stretch"])
            qk = rng.choice([1, 2, 4, 8])
            case = _delta(dtype, _log_int(rng, 1, COARSE if form == "cells" else 8),
                          rng.choice([1, 1, 1, 2, 5, 16]) if form == "cells" else _log_int(rng, 17, 10 * COARSE),
                          qk * rng.choice([1, 1, 2]), rng.choice([32, 64, 128]), rng.choice([32, 64, 128]), qk_heads=qk,
                          ragged=rng.random() < 0.5)
        if _cost(case) <= most[op] and work(case)["bytes"] < 1.5e9:
            return case


def _lengths(case):
    """Queries and keys (cross), or new tokens (delta), of every sequence."""
    batch = case["batch"]
    sizes = [case["queries"], case["keys"]] if case["op"] == "cross" else [case["new"]]
    if not case["ragged"]:
        out = [[n] * batch for n in sizes]
    else:
        rng = random.Random(batch * 1000003 + sizes[0] * 1009 + sizes[-1])
        out = [[n] + [rng.randint(min(1, n // 4), n) for _ in range(batch - 1)] for n in sizes]
    return out if case["op"] == "cross" else out[0]


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _starts(lengths):
    return torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    """The tensors of a case on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = _dtype(case)

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std + mean).to(kind)

    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        s = dict(x=normal(rows, width, std=2.0, mean=0.3), weight=normal(width, std=0.2, mean=1.0))
        if case["bias"]:
            s["bias"] = normal(width, std=0.2)
        if case["block"]:
            s["block"] = normal(rows, width, std=0.7)
            if case["post"]:
                s["block_weight"] = normal(width, std=0.2, mean=1.0)
                if case["bias"]:
                    s["block_bias"] = normal(width, std=0.2)
            if case["scale"]:
                s["scale"] = normal(width, std=0.1, mean=0.3)
        if case["gate"] == "row":
            s["gate"] = normal(rows, width)
        elif case["gate"] == "image":
            s["gate"] = normal(case["images"], width)
        return s
    if case["op"] == "cross":
        queries, keys = _lengths(case)
        heads, kv, dim, nq, nk = case["q_heads"], case["kv_heads"], case["dim"], sum(queries), sum(keys)
        # a normalised query's logits: standard deviation 2
        s = dict(q=normal(nq, heads, dim, std=2.0))
        if case["fused"]:
            both = normal(nk, 2, kv, dim)
            s["k"], s["v"] = both[:, 0], both[:, 1]
        else:
            s["k"], s["v"] = normal(nk, kv, dim), normal(nk, kv, dim)
        if case["visible"] < 1:
            # occupied cells come in runs along a row of the map
            run = 4
            seen = torch.rand(-(-nk // run), generator=gen, device="cuda") < case["visible"]
            s["mask"] = seen.repeat_interleave(run)[:nk].contiguous()
            if case["ragged"] and case["batch"] > 1:
                s["mask"][keys[0]:keys[0] + keys[1]] = False
        if case["ragged"]:
            s["q_start"], s["k_start"] = _starts(queries), _starts(keys)
        return s
    new = _lengths(case)
    total, heads, qk, dk, dv = sum(new), case["heads"], case["qk_heads"], case["key_dim"], case["value_dim"]
    # queries, keys, values and the two gates are columns of one projection's rows
    rows = normal(total, 2 * qk * dk + heads * dv + 2 * heads)
    s = dict(rows=rows, state=torch.randn(case["batch"], heads, dk, dv, generator=gen, device="cuda") * 0.3)
    at = 0
    for name, n, d in (("q", qk, dk), ("k", qk, dk), ("v", heads, dv), ("a", heads, 0), ("b", heads, 0)):
        part = rows[:, at:at + n * max(d, 1)]
        s[name] = part.unflatten(1, (n, d)) if d else part
        at += n * max(d, 1)
    # heads that forget within some ten tokens and heads that hold on for thousands
    s["rate"] = torch.exp(torch.rand(heads, generator=gen, device="cuda") * math.log(16.0))
    s["bias"] = torch.rand(heads, generator=gen, device="cuda") * 5.0 - 7.0
    s["start"] = _starts(new)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own and case["op"] == "delta":
        import paper_2512_08557_amd as ssc
        s["memory"] = ssc.DeltaMemory(case["batch"], case["heads"], case["key_dim"], case["value_dim"],
                                      qk_heads=case["qk_heads"], dtype=case["dtype"])
    return s


def run(state):
    case = state["case"]
    return {"norm": _run_norm, "cross": _run_cross, "delta": _run_delta}[case["op"]](state, case)


def _normed(x, weight, bias, center):
    if center:
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    if weight is not None:
        x = x * weight.float()
    return x if bias is None else x + bias.float()


def _gated(x, s, case):
    if case["gate"] == "none":
        return x
    g = s["gate"].float()
    if case["act"] != "none":
        sig = 1 / (1 + torch.exp(-g))
        g = sig if case["act"] == "sigmoid" else g * sig
    if case["gate"] == "image":
        return (x.view(case["images"], -1, case["width"]) * g[:, None]).view(-1, case["width"])
    return x * g


def _run_norm(s, case):
    act = None if case["act"] == "none" else case["act"]
    if own:
        import paper_2512_08557_amd as ssc
        x, gate = s["x"], s.get("gate")
        if case["gate"] == "image":
            x = x.view(case["images"], -1, case["width"])
        if not case["block"]:
            return ssc.norm(x, s["weight"], s.get("bias"), eps=EPS, center=case["center"], gate=gate,
                            activation=act).view(-1, case["width"])
        total, y = ssc.add_norm(x, s["block"].view(x.shape), s["weight"], s.get("bias"),
                                block_weight=s.get("block_weight"), block_bias=s.get("block_bias"), gate=gate,
                                activation=act, scale=s.get("scale"), eps=EPS, center=case["center"])
        return total.view(-1, case["width"]), y.view(-1, case["width"])
    x = s["x"].float()
    if not case["block"]:
        return _gated(_normed(x, s["weight"], s.get("bias"), case["center"]), s, case).to(_dtype(case))
    z = s["block"].float()
    if case["post"]:
        z = _normed(z, s["block_weight"], s.get("block_bias"), case["center"])
    z = _gated(z, s, case)
    if case["scale"]:
        z = z * s["scale"].float()
    z = x + z
    return z.to(_dtype(case)), _normed(z, s["weight"], s.get("bias"), case["center"]).to(_dtype(case))


def _run_cross(s, case):
    queries, keys = _lengths(case)
    if own:
        import paper_2512_08557_amd as ssc
        if case["ragged"]:
            return ssc.cross_attend(s["q"], s["k"], s["v"], mask=s.get("mask"), q_start=s["q_start"],
                                    k_start=s["k_start"], max_q=case["queries"], max_k=case["keys"])
        dense = [s[n].unflatten(0, (case["batch"], -1)) if n in s else None for n in ("q", "k", "v", "mask")]
        return ssc.cross_attend(*dense).flatten(0, 1)
    kv, group = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    out, q0, k0 = [], 0, 0
    for nq, nk in zip(queries, keys):
        if nk == 0:
            out.append(s["q"].new_zeros(nq, *s["q"].shape[1:]))
            q0 += nq
            continue
        k = s["k"][k0:k0 + nk].float().permute(1, 2, 0).contiguous()
        v = s["v"][k0:k0 + nk].float().transpose(0, 1).contiguous()
        seen = s["mask"][k0:k0 + nk] if "mask" in s else None
        if seen is not None:
            v = torch.where(seen[:, None], v, torch.zeros_like(v))
        # as many queries at once as keep the scores within 4 GB
        step = max(1, 2 ** 30 // max(1, nk * case["q_heads"]))
        for i in range(0, nq, step):
            n = min(step, nq - i)
            x = s["q"][q0 + i:q0 + i + n].float().view(n, kv, group, -1).permute(1, 2, 0, 3).reshape(kv, group * n, -1)
            score = torch.matmul(x, k).mul_(1 / math.sqrt(case["dim"]))
            if seen is not None:
                score.masked_fill_(~seen, -math.inf)
            top = score.amax(-1, keepdim=True)
            score = score.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
            total = score.sum(-1, keepdim=True)
            y = torch.matmul(score, v)
            y = torch.where(total == 0, torch.zeros_like(y), y / total).view(kv, group, n, -1)
            out.append(y.permute(2, 0, 1, 3).reshape(n, kv * group, -1).to(_dtype(case)))
        q0, k0 = q0 + nq, k0 + nk
    return torch.cat(out)


def _padded(s, case):
    """Queries, keys and values [batch, heads, tokens, dim], the logarithm of alpha (64 bits) and beta [batch,
    heads, tokens], and where the call's rows are among them; a stream's missing tokens change nothing."""
    new = _lengths(case)
    most = case["new"] if case["new"] <= CHUNK else -(-case["new"] // CHUNK) * CHUNK
    row, at = torch.arange(sum(new), device="cuda"), s["start"].long()
    seq = torch.searchsorted(at[1:].contiguous(), row, right=True)
    place = seq * most + row - at[seq]

    def spread(x, heads):
        x = x.repeat_interleave(case["heads"] // heads, 1)
        y = torch.zeros(case["batch"] * most, *x.shape[1:], dtype=x.dtype, device="cuda")
        y[place] = x
        return y.unflatten(0, (case["batch"], most)).transpose(1, 2).contiguous()

    q, k = s["q"].float(), s["k"].float()
    q = q * torch.rsqrt((q * q).sum(-1, keepdim=True) + EPS) * (1 / math.sqrt(case["key_dim"]))
    k = k * torch.rsqrt((k * k).sum(-1, keepdim=True) + EPS)
    a = s["a"].double() + s["bias"].double()
    g = -s["rate"].double() * torch.where(a > 30, a, torch.log1p(torch.exp(a)))
    beta = 1 / (1 + torch.exp(-s["b"].float()))
    return (spread(q, case["qk_heads"]), spread(k, case["qk_heads"]), spread(s["v"].float(), case["heads"]),
            spread(g, case["heads"]), spread(beta, case["heads"]), place)


def _run_delta(s, case):
    if own:
        memory = s["memory"]
        out = memory.update(s["q"], s["k"], s["v"], s["a"], s["b"], rate=s["rate"], bias=s["bias"], eps=EPS,
                            start=s["start"], max_new=case["new"], initial=s["state"])
        return out, memory.state
    q, k, v, g, beta, place = _padded(s, case)
    S, tokens = s["state"], q.shape[2]
    if tokens <= CHUNK:
        out = torch.empty_like(v)
        for t in range(tokens):
            key = k[:, :, t, :, None]
            S = S * torch.exp(g[:, :, t]).float()[..., None, None]
            u = beta[:, :, t, None] * (v[:, :, t] - (S * key).sum(-2))
            S = S + key * u[:, :, None]
            out[:, :, t] = (S * q[:, :, t, :, None]).sum(-2)
    else:
        # chunks: a triangular system each, and from one to the next the state alone
        q, k, v, g, beta = (x.unflatten(2, (-1, CHUNK)) for x in (q, k, v, g, beta))
        total = torch.cumsum(g, -1)
        decay = torch.exp(torch.tril(total[..., :, None] - total[..., None, :])).float().tril_()
        since, left = torch.exp(total).float()[..., None], torch.exp(total[..., -1:] - total).float()[..., None]
        kt = k.transpose(-1, -2).contiguous()
        system = torch.matmul(k, kt) * decay * beta[..., None]
        inverse = torch.eye(CHUNK, device="cuda").expand(system.shape).contiguous()
        for i in range(1, CHUNK):
            inverse[..., i, :i] = -torch.matmul(system[..., i:i + 1, :i], inverse[..., :i, :i].contiguous())[..., 0, :]
        W = torch.matmul(inverse, k * (beta[..., None] * since))
        U = torch.matmul(inverse, v * beta[..., None])
        scores = torch.matmul(q, kt) * decay
        q = q * since
        k = (k * left).transpose(-1, -2).contiguous()
        out = torch.empty_like(v)
        for c in range(q.shape[2]):
            u = U[:, :, c] - torch.matmul(W[:, :, c], S)
            out[:, :, c] = torch.matmul(q[:, :, c], S) + torch.matmul(scores[:, :, c], u)
            S = S * since[:, :, c, -1:] + torch.matmul(k[:, :, c], u)
        out = out.flatten(2, 3)
    out = out.transpose(1, 2).flatten(0, 1)[place]
    return out.to(_dtype(case)), S


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        full = (4 if case["block"] else 2) + (1 if case["gate"] == "row" else 0)
        small = 1 + case["bias"] + (case["block"] and case["post"]) * (1 + case["bias"]) + \
            (case["block"] and case["scale"]) + (case["images"] if case["gate"] == "image" else 0)
        return {"bytes": size * width * (rows * full + small), "flops": 12.0 * rows * width}
    if case["op"] == "cross":
        queries, keys = _lengths(case)
        heads, kv, dim, share = case["q_heads"], case["kv_heads"], case["dim"], case["visible"]
        if case["ragged"] and share < 1 and case["batch"] > 1:
            keys = [0 if i == 1 else n for i, n in enumerate(keys)]
        return {"bytes": size * dim * (2 * sum(queries) * heads + 2 * kv * share * sum(keys)) +
                (sum(keys) if share < 1 else 0),
                "flops": 4.0 * heads * dim * share * sum(m * n for m, n in zip(queries, keys))}
    total, heads, qk, dk, dv = sum(_lengths(case)), case["heads"], case["qk_heads"], case["key_dim"], case["value_dim"]
    return {"bytes": size * total * (2 * qk * dk + 2 * heads * dv + 2 * heads) + 8 * case["batch"] * heads * dk * dv,
            "flops": 7.0 * total * heads * dk * dv}


def exact(case, seed):
    """The operators by their definitions in 64 bits."""
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "cross": _exact_cross, "delta": _exact_delta}[case["op"]](s, case)


def _exact_norm(s, case):
    def one(x, weight, bias):
        if case["center"]:
            x = x - x.sum(-1, keepdim=True) / x.shape[-1]
        x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
        return x if bias is None else bias.double() + x

    sums, outs = [], []
    for rows in torch.split(torch.arange(case["rows"], device="cuda"), 65536):
        z = s["block" if case["block"] else "x"][rows].double()
        if not case["block"]:
            z = one(z, s["weight"], s.get("bias"))
        elif case["post"]:
            z = one(z, s["block_weight"], s.get("block_bias"))
        if case["gate"] != "none":
            g = s["gate"][rows if case["gate"] == "row" else rows // (case["rows"] // case["images"])].double()
            z = z * {"none": lambda t: t, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu}[case["act"]](g)
        if not case["block"]:
            outs.append(z)
            continue
        if case["scale"]:
            z = z * s["scale"].double()
        sums.append(s["x"][rows].double() + z)
        outs.append(one(sums[-1], s["weight"], s.get("bias")))
    return (torch.cat(sums), torch.cat(outs)) if case["block"] else torch.cat(outs)


def _exact_cross(s, case):
    if work(case)["flops"] > 5e12:
        return None
    queries, keys = _lengths(case)
    out = torch.zeros(sum(queries), case["q_heads"], case["dim"], dtype=torch.float64, device="cuda")
    q0 = k0 = 0
    for nq, nk in zip(queries, keys):
        here = torch.arange(k0, k0 + nk, device="cuda")
        if "mask" in s:
            here = here[s["mask"][here]]
        if len(here):
            for h in range(case["q_heads"]):
                g = h * case["kv_heads"] // case["q_heads"]
                keys_h, values_h = s["k"][here, g].double(), s["v"][here, g].double()
                for at in torch.split(torch.arange(q0, q0 + nq, device="cuda"), 1024):
                    z = torch.mm(s["q"][at, h].double(), keys_h.t()) / math.sqrt(case["dim"])
                    out[at, h] = torch.mm(torch.softmax(z, -1), values_h)
        q0, k0 = q0 + nq, k0 + nk
    return out


def _exact_delta(s, case):
    new, heads, dk = _lengths(case), case["heads"], case["key_dim"]
    which = torch.arange(heads, device="cuda") * case["qk_heads"] // heads
    S = s["state"].double()
    out = torch.zeros(sum(new), heads, case["value_dim"], dtype=torch.float64, device="cuda")

    def unit(x):
        x = x.double()
        return x / torch.sqrt((x ** 2).sum(-1, keepdim=True) + EPS)

    alpha = torch.exp(-s["rate"].double() * torch.nn.functional.softplus(s["a"].double() + s["bias"].double(), threshold=40))
    beta = torch.sigmoid(s["b"].double())
    first = [0] + list(np.cumsum(new))
    # the streams by length, so that the ones with a token left come first
    order = sorted(range(case["batch"]), key=lambda b: -new[b])
    begin = torch.tensor([first[b] for b in order], device="cuda")
    S = S[torch.tensor(order, device="cuda")]
    live = len(order)
    for t in range(max(new)):
        while live and new[order[live - 1]] <= t:
            live -= 1
        at = begin[:live] + t
        k, q = unit(s["k"][at])[:, which, :, None], unit(s["q"][at])[:, which, None]
        T = S[:live] * alpha[at][..., None, None]
        miss = s["v"][at].double() - torch.matmul(k.transpose(-1, -2).contiguous(), T)[..., 0, :]
        T = T + k * (beta[at][..., None] * miss)[..., None, :]
        S[:live] = T
        out[at] = torch.matmul(q, T)[..., 0, :] / math.sqrt(dk)
    back = torch.empty_like(S)
    back[torch.tensor(order, device="cuda")] = S
    return out, back
