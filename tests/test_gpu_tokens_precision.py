"""GPU tests of how near the token operators come to 64 bits where a looser
bound would hide a fault."""
import math

import numpy as np
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2512_08557_amd as ssc  # noqa: E402

U = 2.0 ** -24


def normal(rng, shape, kind, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(kind).cuda()


@pytest.mark.parametrize("batch,heads,kv,dim,keys", [(1, 1, 1, 32, 1), (4, 8, 2, 64, 4096), (2, 4, 4, 128, 777),
                                                     (3, 16, 1, 32, 5000), (2, 32, 1, 64, 65), (1, 8, 8, 128, 20000)])
def test_single_bf16_tokens_are_off_by_the_rounding_of_the_output_alone(batch, heads, kv, dim, keys):
    """Scores: 2 (sqrt(D) + 8) u scale sum |q k| and 4 u of themselves before exp,
    twice (numerator and sum); sums of `keys` terms 2 (sqrt(keys) + 8) u; a
    probability in two bf16 parts is off by 2^-8 of what the first leaves, itself
    2^-8 of the value: 2^-16; all relative to sum p |v|.  Then the output's
    rounding, 2^-8 at most, and 2 u."""
    note(f"[gpu-test] single bf16 tokens {batch} {heads} {kv} {dim} {keys}")
    rng = np.random.default_rng(keys + dim)
    kind = torch.bfloat16
    k, v = (normal(rng, (batch, kv, keys, dim), kind) for _ in range(2))
    c = ssc.TokenCache(batch, kv, dim, keys, dtype="bf16", k=k, v=v)
    c.seek([keys - 1] * batch)
    q = normal(rng, (batch, heads, dim), kind, 2.0)
    got = c.attend(q, keys).double().cpu()
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    worst = 0.0
    for b in range(batch):
        for h in range(heads):
            kk, vv, x = k[b, h * kv // heads], v[b, h * kv // heads], q[b, h]
            s = kk @ x / math.sqrt(dim)
            p = torch.softmax(s, 0)
            ref = p @ vv
            err = 2 * (math.sqrt(dim) + 8) * U * (kk.abs() @ x.abs()) / math.sqrt(dim) + 4 * U * s.abs()
            rel = 2 * float(err.max()) + 2 * (math.sqrt(keys) + 8) * U + 2.0 ** -16
            tol = rel * (p @ vv.abs()) + (2.0 ** -8 + 2 * U) * ref.abs()
            worst = max(worst, float(((got[b, h] - ref).abs() / tol).max()))
    note(f"[gpu-test] {worst:.3f} of the tolerance")
    assert worst <= 1.0


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 40, 150])
@pytest.mark.parametrize("scale", [1e-32, 0.0, -1e-32])
def test_tiny_scales(kind, new, scale):
    """Scores whose scale is far below one and whose products are as large.
    Tolerance: as for attention in general, 2^-8 for every bf16 probability and
    the output."""
    note(f"[gpu-test] scale {scale} {kind} new {new}")
    rng = np.random.default_rng(new)
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    k, v = normal(rng, (1, 1, 200, 32), dtype, 1e16), normal(rng, (1, 1, 200, 32), dtype)
    c = ssc.TokenCache(1, 1, 32, 200, dtype=kind, k=k, v=v)
    c.seek([200 - new])
    q = normal(rng, (new, 1, 32), dtype, 1e15)
    got = c.attend(q, 200, causal=False, scale=scale)[:, 0].double().cpu()
    q, k, v = q[:, 0].double().cpu(), k[0, 0].double().cpu(), v[0, 0].double().cpu()
    s = scale * (q @ k.t())
    p = torch.softmax(s, -1)
    err = 2 * (math.sqrt(32) + 8) * U * abs(scale) * (q.abs() @ k.abs().t()) + 4 * U * s.abs()
    rel = 2 * err.max(-1, keepdim=True)[0] + 2 * (math.sqrt(200) + 8) * U + (2.0 ** -8 if kind == "bf16" else 0)
    tol = rel * (p @ v.abs()) + (2.0 ** -8 * (kind == "bf16") + 2 * U) * (p @ v).abs()
    assert bool(((got - p @ v).abs() <= tol).all()), float(((got - p @ v).abs() / tol).max())


@pytest.mark.parametrize("rows", [50, 20000])
def test_gelu_tends_to_zero(rows):
    """z Phi(z) of z = x (one channel, weight 1).  Everywhere within 4 u |z| (the
    polynomial 1.7e-8, its evaluation and the exponential 2.5 u, the sum u); from
    z = -6 downwards no further from zero than a tenth above the function itself
    (the polynomial lies below log2 Phi there), and zero at minus infinity."""
    note(f"[gpu-test] gelu tail {rows}")
    z = torch.linspace(-45, 12, rows)
    z[0], z[1], z[-1], z[2] = -math.inf, -3e38, math.inf, -1000.0
    y = ssc.linear(z[:, None].cuda(), torch.ones(1, 1, device="cuda"), activation="gelu")[:, 0].double().cpu()
    assert y[0] == 0 and y[1] == 0 and y[2] == 0 and y[-1] == math.inf
    z, y = z.double()[3:-1], y[3:-1]
    ref = 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    assert bool(((y - ref).abs() <= 4 * U * z.abs() + 1e-45).all()), float(((y - ref).abs() / (4 * U * z.abs())).max())
    tail = z <= -6
    assert bool((y[tail].abs() <= 1.1 * ref[tail].abs()).all()), float((y[tail] / ref[tail]).abs().max())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [20, 20000])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_activations_keep_nan_and_infinity(act, rows, kind):
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    x = torch.ones(rows, 8, dtype=dtype, device="cuda")
    x[1, 2], x[rows - 1, 0], x[3, 1] = math.nan, math.nan, math.inf
    y = ssc.linear(x, torch.ones(128, 8, dtype=dtype, device="cuda"), activation=act)
    lost = torch.isnan(y).all(1).cpu()
    assert lost[1] and lost[rows - 1] and int(lost.sum()) == 2 and int(torch.isnan(y).sum()) == 256
    assert bool((y[3] == math.inf).all()) and int(torch.isinf(y).sum()) == 128
