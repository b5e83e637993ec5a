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
