"""GPU tests of norms in which the same lanes take several rows one after the other, with
gates that change within such a run.

Tolerances as in test_gpu_norms.py, whose norm in 64 bits (with how far fp32 may be from
it) this file uses; a gate is off by 16 u, a product or sum by u = 2^-24 of itself, an
output by 2 u, in bf16 by 2^-8 and 2 u of itself."""
import numpy as np
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2512_08557_amd as ssc  # noqa: E402
from test_gpu_norms import KIND, OUT, U, normal, normed  # noqa: E402


def close(got, ref, tol, what):
    worst = float(((got.double() - ref).abs() / (tol + 1e-37)).max())
    note(f"[gpu-test] {what}: {worst:.3f} of the tolerance")
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


def gate_of(gate, act, shape):
    g = gate.double()
    g = {None: g, "silu": g * torch.sigmoid(g), "sigmoid": torch.sigmoid(g)}[act]
    return g.view(gate.shape[:-1] + (1,) * (len(shape) - gate.dim()) + gate.shape[-1:])


# rows of a gate that end within a run, several of them within one, the last run cut short; widths with a rest
SHAPES = [((3, 22003, 384), 1), ((40001, 3, 384), 1), ((12001, 3, 512), 1), ((7001, 5, 512), 1), ((5, 7001, 500), 1),
          ((30001, 512), 0), ((30001, 512), 1), ((11, 2749, 3, 509), 2), ((4099, 7, 1100), 1)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape,lead", SHAPES)
def test_gates_that_change_within_a_run(shape, lead, kind):
    note(f"[gpu-test] norms of {shape}, a gate of {shape[:lead]}, {kind}")
    rng = np.random.default_rng(shape[-1] + shape[0])
    k = KIND[kind]
    x, block = (normal(rng, shape, k, 1.0, 0.3) for _ in range(2))
    gate = normal(rng, shape[:lead] + shape[-1:], k, 2.0)
    w, b, bw, bb, scale = (normal(rng, shape[-1:], k, 0.3, m) for m in (1, 0, 1, 0, 0.5))
    for act, center, post, scaled in (("silu", True, True, True), ("sigmoid", False, False, False)):
        total, out = ssc.add_norm(x, block, w, b, block_weight=bw if post else None, block_bias=bb if post else None, gate=gate,
                                  activation=act, scale=scale if scaled else None, center=center)
        z = block.double()
        tol = torch.zeros_like(z)
        if post:
            z, tol = normed(z, tol, bw.double(), bb.double(), center, 1e-6)
        g = gate_of(gate, act, shape)
        z, tol = z * g, tol * g.abs() + 16 * U * (z * g).abs()
        if scaled:
            z, tol = z * scale.double(), (tol + U * z.abs()) * scale.double().abs()
        z = z + x.double()
        tol = tol + U * z.abs()
        close(total, z, tol + OUT[kind] * z.abs(), f"total {act}")
        y, tol = normed(z, tol, w.double(), b.double(), center, 1e-6)
        close(out, y, tol + OUT[kind] * y.abs(), f"out {act}")
    got = ssc.norm(x, w, b, center=True, gate=gate, activation="silu")
    y, tol = normed(x.double(), torch.zeros(shape, dtype=torch.float64, device="cuda"), w.double(), b.double(), True, 1e-6)
    g = gate_of(gate, "silu", shape)
    y, tol = y * g, tol * g.abs() + 16 * U * (y * g).abs()
    close(got, y, tol + OUT[kind] * y.abs(), "norm")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_runs_in_place(kind):
    """The next row's values are under way while this one's are written."""
    rng = np.random.default_rng(2)
    x, block = (normal(rng, (3, 22003, 384), KIND[kind]) for _ in range(2))
    gate, w = normal(rng, (3, 384), KIND[kind]), normal(rng, (384,), KIND[kind])
    want = ssc.add_norm(x, block, w, gate=gate, activation="silu")
    a, b = x.clone(), block.clone()
    ssc.add_norm(a, b, w, gate=gate, activation="silu", total=a, out=b)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    y = ssc.norm(x, w, gate=block)
    assert torch.equal(ssc.norm(x, w, gate=block, out=block), y)
