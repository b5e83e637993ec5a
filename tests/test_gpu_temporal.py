"""GPU test of the temporal block on a backbone's map: Engine, linear, append,
attend and advance as they run together, against the block in 64 bits.

Tolerance: the operators' own are tested by themselves; here one stride's error
passes through four layers and a softmax.  In fp32 every intermediate is off by
some ten roundings of sums of up to 512 terms (2 sqrt(512) 2^-24 = 2.7e-6 of the
size of the terms); through scores of size up to ten and three more layers a
hundred times that, 3e-4 of the largest output, is a wide bar that any wrong
mask, position or slot exceeds.  bf16 rounds six intermediates to 2^-8 each:
6 * 2^-8 = 2.3e-2 of the largest."""
import numpy as np
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2512_08557_amd import Engine, TemporalBlock, linear  # noqa: E402

H = W = 40
C, HEADS, KV, DIM, INNER, STRIDES, SINKS = 64, 4, 2, 32, 192, 3, 5


def reference(w, maps, grid):
    """The block's result for the last of the strides seen so far, in 64 bits."""
    w = {k: v.double().cpu() for k, v in w.items()}
    h, wd = grid
    n = h * wd
    rows, cols = torch.meshgrid(torch.arange(h), torch.arange(wd), indexing="ij")
    sec = (DIM // 4, DIM // 8, DIM // 8)
    freq = torch.cat([10000.0 ** (-torch.arange(s, dtype=torch.float64) / s) for s in sec]).float().double()

    def turned(x, weight, stride):
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
        pos = torch.stack([torch.full((n,), stride), rows.flatten(), cols.flatten()], 1).double()
        t = torch.cat([pos[:, i:i + 1].expand(n, s) for i, s in enumerate(sec)], 1) * freq
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        a, b = x[..., :DIM // 2], x[..., DIM // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    ks, vs = [], []
    for i, x in enumerate(maps):
        z = (x @ w["qkv"].t() + w["qkv_bias"]).view(n, HEADS + 2 * KV, DIM)
        ks.append(turned(z[:, HEADS:HEADS + KV], w["k_norm"], i))
        vs.append(z[:, HEADS + KV:])
    q = turned(z[:, :HEADS], w["q_norm"], len(maps) - 1)
    k, v = torch.cat(ks), torch.cat(vs)
    past = (len(maps) - 1) * n
    j = torch.arange(past + n)
    seen = (j >= past - STRIDES * n) | (j < SINKS)
    out = torch.empty(n, HEADS, DIM, dtype=torch.float64)
    for g in range(HEADS):
        kk, vv = k[seen][:, g * KV // HEADS], v[seen][:, g * KV // HEADS]
        out[:, g] = torch.softmax(q[:, g] @ kk.t() / DIM ** 0.5, -1) @ vv
    y = maps[-1] + out.reshape(n, -1) @ w["out"].t()
    u = y @ w["up"].t() + w["up_bias"]
    u = 0.5 * u * torch.special.erfc(-u / 2 ** 0.5)
    z = y + u @ w["down"].t()
    return z @ w["head"].t() + w["head_bias"]


@pytest.mark.parametrize("dtype,bar", [("f32", 3e-4), ("bf16", 2.3e-2)])
def test_temporal_block_over_a_backbone(dtype, bar):
    rng = np.random.default_rng(21)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    bits = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(kind)  # noqa: E731
    conv = [bits(rng.standard_normal((64, 64, 3, 3)) * (2 / 576) ** 0.5) for _ in range(2)]
    eng = Engine(H, W, 64, [(64, 64, 2, True), (64, 64, 2, True)], [t.float().numpy() for t in conv], dtype=dtype,
                 max_pillars=600)
    grid = eng.shapes[2][:2]
    n = grid[0] * grid[1]
    make = lambda *s: bits(rng.standard_normal(s) * s[-1] ** -0.5).cuda()  # noqa: E731
    w = {"qkv": make((HEADS + 2 * KV) * DIM, C), "qkv_bias": make((HEADS + 2 * KV) * DIM), "q_norm": make(DIM) + 1,
         "k_norm": make(DIM) + 1, "out": make(C, HEADS * DIM), "up": make(INNER, C), "up_bias": make(INNER),
         "down": make(C, INNER), "head": make(42, C), "head_bias": make(42)}
    block = TemporalBlock(w, HEADS, KV, DIM, tokens=n, strides=STRIDES, sinks=SINKS)
    for run in range(2):
        maps = []
        for stride in range(7 if run == 0 else 2):
            idx = np.sort(rng.choice(H * W, 400, replace=False)).astype(np.int32)
            feats = bits(rng.standard_normal((400, 64))).cuda()
            eng.step(torch.from_numpy(idx).cuda(), feats, sorted=True)
            x = eng.read(2).view(-1, C)
            maps.append(x.double().cpu())
            out = linear(block.step(x, stride, grid), w["head"], w["head_bias"])
            ref = reference(w, maps, grid)
            err = float((out.double().cpu() - ref).abs().max() / ref.abs().max())
            note(f"[gpu-test] temporal block {dtype} run {run} stride {stride}: {err:.2e}")
            assert err <= bar, f"stride {stride}: {err}"
        assert block.cache.past.tolist() == [len(maps) * n]
        block.reset()
    eng.close()


def test_missing_weights_are_refused():
    with pytest.raises(ValueError, match="down"):
        TemporalBlock({"qkv": 0, "q_norm": 0, "k_norm": 0, "out": 0, "up": 0}, 4, 2, 32, 16, 2)
