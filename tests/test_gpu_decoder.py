"""GPU test of the query decoder on a backbone's map: Engine, norms, delta memory,
cross attention and linear layers as they run together, against 64 bits.

Tolerance as for the temporal block: in fp32 every intermediate is off by some ten
roundings of sums of up to 512 terms (2 sqrt(512) 2^-24 = 2.7e-6 of the size of the
terms); through norms, scores of size up to ten and eight more layers a hundred times
that, 3e-4 of the largest output, is a wide bar that any wrong mask, stream or column
exceeds.  bf16 rounds eleven intermediates of the residual stream to half a step, 2^-9
each, which feed one another through norms, and the delta memory carries those of
the strides before: 11 * 2 * 2^-9 = 4.3e-2 of the largest."""
import numpy as np
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2512_08557_amd import Engine, QueryDecoder  # noqa: E402

H = W = 40
CELLS, C, QUERIES, MH, QK, DK, DV, QH, KV, DIM, INNER = 64, 96, 50, 4, 2, 32, 64, 4, 2, 32, 192


def make_weights(rng, kind):
    make = lambda *s: torch.from_numpy((rng.standard_normal(s) * s[-1] ** -0.5).astype(np.float32)).to(kind).cuda()  # noqa: E731
    one = lambda n: (1 + 0.2 * make(n, 1).view(n)).to(kind)  # noqa: E731
    return {"norm": one(C), "cross_norm": one(C), "ffn_norm": one(C), "out_norm": one(C), "memory_norm": one(DV),
            "memory": make(2 * QK * DK + MH * DV + 2 * MH, C), "memory_gate": make(MH * DV, C), "memory_out": make(C, MH * DV),
            "q": make(QH * DIM, C) * 2, "kv": make(2 * KV * DIM, CELLS), "kv_bias": make(2 * KV * DIM, 1).view(-1),
            "cross_out": make(C, QH * DIM), "cross_scale": one(C), "up": make(INNER, C), "up_bias": make(INNER, 1).view(-1),
            "down": make(C, INNER), "rate": torch.rand(MH, device="cuda") + 0.5, "bias": torch.rand(MH, device="cuda") - 3}


def reference(w, S, x, cells, seen):
    """One stride of one image in 64 bits: the state, x and the norm after it."""
    def rms(t, weight):
        return t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * weight

    n = x.shape[0]
    h = rms(x, w["norm"])
    q, k, v, a, b = (h @ w["memory"].t()).split([QK * DK, QK * DK, MH * DV, MH, MH], 1)
    q, k = (t.view(n, QK, DK) / torch.sqrt((t.view(n, QK, DK) ** 2).sum(-1, keepdim=True) + 1e-6) for t in (q, k))
    q, k = q.repeat_interleave(MH // QK, 1), k.repeat_interleave(MH // QK, 1)
    alpha = torch.exp(-w["rate"] * torch.nn.functional.softplus(a + w["bias"]))[..., None]
    S = S * alpha[..., None]
    u = torch.sigmoid(b)[..., None] * (v.view(n, MH, DV) - (S * k[..., None]).sum(2))
    S = S + k[..., None] * u[:, :, None]
    o = (S * q[..., None]).sum(2) * DK ** -0.5
    o = rms(o, w["memory_norm"]) * torch.nn.functional.silu((h @ w["memory_gate"].t()).view(n, MH, DV))
    x = x + o.reshape(n, -1) @ w["memory_out"].t()
    h = rms(x, w["cross_norm"])
    q = (h @ w["q"].t()).view(n, QH, DIM)
    kv = (cells[seen] @ w["kv"].t() + w["kv_bias"]).view(-1, 2, KV, DIM)
    c = torch.zeros(n, QH, DIM, dtype=torch.float64)
    for g in range(QH if len(kv) else 0):
        c[:, g] = torch.softmax(q[:, g] @ kv[:, 0, g * KV // QH].t() * DIM ** -0.5, -1) @ kv[:, 1, g * KV // QH]
    x = x + w["cross_scale"] * (c.reshape(n, -1) @ w["cross_out"].t())
    u = rms(x, w["ffn_norm"]) @ w["up"].t() + w["up_bias"]
    x = x + (0.5 * u * torch.special.erfc(-u / 2 ** 0.5)) @ w["down"].t()
    return S, x, rms(x, w["out_norm"])


@pytest.mark.parametrize("dtype,bar", [("f32", 3e-4), ("bf16", 4.3e-2)])
def test_query_decoder_over_a_backbone(dtype, bar):
    rng = np.random.default_rng(31)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    bits = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(kind)  # noqa: E731
    conv = [bits(rng.standard_normal((64, 64, 3, 3)) * (2 / 576) ** 0.5) for _ in range(2)]
    eng = Engine(H, W, 64, [(64, 64, 2, True), (64, 64, 2, True)], [t.float().numpy() for t in conv], dtype=dtype,
                 max_pillars=600)
    w = make_weights(rng, kind)
    exact = {k: v.double().cpu() for k, v in w.items()}
    dec = QueryDecoder(w, QUERIES, MH, DK, DV, QH, KV, DIM, qk_heads=QK, batch=2)
    begin = bits(rng.standard_normal((2, QUERIES, C))).cuda()
    for run in range(2):
        x = begin
        S = [torch.zeros(QUERIES, MH, DK, DV, dtype=torch.float64) for _ in range(2)]
        for stride in range(5 if run == 0 else 2):
            idx = np.sort(rng.choice(H * W, 400, replace=False)).astype(np.int32)
            eng.step(torch.from_numpy(idx).cuda(), bits(rng.standard_normal((400, 64))).cuda(), sorted=True)
            one = eng.read(2).view(1, -1, CELLS)
            cells = torch.cat([one, one.flip(1)])
            mask = torch.from_numpy(rng.random((2, cells.shape[1])) < 0.4).cuda()
            mask[1] &= stride != 1                     # an image without a cell
            before = x.double().cpu()
            x, y = dec.step(x, cells, mask if stride != 2 else None)
            for b in range(2):
                seen = mask[b].cpu() if stride != 2 else slice(None)
                S[b], rx, ry = reference(exact, S[b], before[b], cells[b].double().cpu(), seen)
                for name, got, ref in (("x", x[b], rx), ("norm", y[b], ry)):
                    err = float((got.double().cpu() - ref).abs().max() / ref.abs().max())
                    note(f"[gpu-test] decoder {dtype} run {run} stride {stride} image {b} {name}: {err:.2e}")
                    assert err <= bar, f"stride {stride} image {b} {name}: {err}"
        dec.reset()
    eng.close()


def test_a_refused_stride_leaves_the_memory():
    w = make_weights(np.random.default_rng(2), torch.float32)
    dec = QueryDecoder(w, QUERIES, MH, DK, DV, QH, KV, DIM, qk_heads=QK)
    x, cells = torch.randn(1, QUERIES, C, device="cuda"), torch.randn(1, 70, CELLS, device="cuda")
    dec.step(x, cells)
    state = dec.memory.state.clone()
    for bad in (lambda: dec.step(x[:, 1:], cells), lambda: dec.step(x, cells[..., 1:]), lambda: dec.step(x, cells[0]),
                lambda: dec.step(x, cells, torch.ones(1, 71, dtype=torch.bool, device="cuda")),
                lambda: dec.step(x, cells, torch.ones(1, 70, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
        assert torch.equal(dec.memory.state, state)


def test_weights_that_a_later_call_would_refuse():
    """A weight behind the memory's: refused when the decoder is made or before the memory is changed."""
    w = make_weights(np.random.default_rng(6), torch.float32)
    args = (QUERIES, MH, DK, DV, QH, KV, DIM)
    wide = torch.ones(C, 2, device="cuda")
    for bad, name in (({"out_norm": wide[:, 0]}, "out_norm"), ({"down": w["down"].t().contiguous().t()}, "down"),
                      ({"up": w["up"].cpu()}, "up"), ({"rate": w["rate"].double()}, "rate")):
        with pytest.raises(ValueError, match=name):
            QueryDecoder(dict(w, **bad), *args, qk_heads=QK)
    dec = QueryDecoder(w, *args, qk_heads=QK)
    x, cells = torch.randn(1, QUERIES, C, device="cuda"), torch.randn(1, 70, CELLS, device="cuda")
    w["down"].requires_grad_(True)
    with pytest.raises(ValueError, match="gradient"):
        dec.step(x, cells)
    assert not bool(dec.memory.state.any())
    with torch.no_grad():
        dec.step(x, cells)
    assert bool(dec.memory.state.any())


def test_captured_strides_replay():
    """A whole stride in a graph: replays go on from stride to stride as eager calls do."""
    rng = np.random.default_rng(4)
    w = make_weights(rng, torch.bfloat16)
    make = lambda: QueryDecoder(w, QUERIES, MH, DK, DV, QH, KV, DIM, qk_heads=QK)  # noqa: E731
    eager, graphed = make(), make()
    data = [(torch.randn(1, 500, CELLS, device="cuda").bfloat16(), torch.rand(1, 500, device="cuda") < 0.3) for _ in range(5)]
    x = begin = torch.randn(1, QUERIES, C, device="cuda").bfloat16()
    want = []
    for cells, mask in data:
        x, y = eager.step(x, cells, mask)
        want.append((x.clone(), y.clone()))
    gx, gc, gm = begin.clone(), data[0][0].clone(), data[0][1].clone()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        x, y = graphed.step(gx, gc, gm)
    torch.cuda.synchronize()
    graphed.reset()
    for i, (cells, mask) in enumerate(data):
        gc.copy_(cells)
        gm.copy_(mask)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want[i][0]) and torch.equal(y, want[i][1]), f"replay {i}"
        gx.copy_(x)
        torch.randn(1000, device="cuda").sum().item()


def test_missing_and_mixed_weights_are_refused():
    w = make_weights(np.random.default_rng(3), torch.float32)
    args = (QUERIES, MH, DK, DV, QH, KV, DIM)
    with pytest.raises(ValueError, match="down"):
        QueryDecoder({k: v for k, v in w.items() if k != "down"}, *args, qk_heads=QK)
    with pytest.raises(ValueError, match="kv_bias"):
        QueryDecoder(dict(w, kv_bias=w["kv_bias"].bfloat16()), *args, qk_heads=QK)
    with pytest.raises(ValueError, match="memory must be"):
        QueryDecoder(w, *args)
