"""GPU tests of norm and add_norm against plain implementations in 64 bits.

Tolerances, from the arithmetic (u = 2^-24): a sum of C fp32 values is off by about
sqrt(C) u of the sum of their sizes, so
  mean    2 (sqrt(C) + 2) u mean|v|
  norm    z / sqrt(mean z^2 + eps) * w + b: half the sum's error in the root and twelve
          roundings, (sqrt(C) + 12) u of the value before b, and what z itself is off by
          (d, of every value) once directly and once through the root, at most
          |d| / |z| in 2-norms of the value
  gate    16 u: an exponential, a quotient, products
  outputs u, in bf16 2^-8 (half a step, 2^-9, twice: a value near a border may fall on
          either side of it in both computations), of themselves
"""
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
KIND = {"f32": torch.float32, "bf16": torch.bfloat16}
OUT = {"f32": 2 * U, "bf16": 2.0 ** -8 + 2 * U}


def normal(rng, shape, kind, std=1.0, mean=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * std + mean).astype(np.float32)).to(kind).cuda()


def close(got, ref, tol, what):
    got = got.double().cpu()
    assert got.shape == ref.shape
    worst = float(((got - ref).abs() / tol.clamp(min=1e-300)).max()) if got.numel() else 0.0
    note(f"[gpu-test] {what}: {worst:.3f} of the tolerance")
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


def normed(z, d, w, b, center, eps):
    """N(z) in 64 bits and how far fp32 may be from it, z being off by d."""
    n = z.shape[-1]
    if center:
        d = d + d.mean(-1, keepdim=True) + 2 * (math.sqrt(n) + 2) * U * z.abs().mean(-1, keepdim=True) + U * z.abs()
        z = z - z.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
    y = z * r
    share = (d.norm(dim=-1, keepdim=True) / z.norm(dim=-1, keepdim=True).clamp(min=math.sqrt(eps * n) + 1e-300)).clamp(max=1)
    tol = d * r + y.abs() * (share + (math.sqrt(n) + 12) * U)
    if w is not None:
        y, tol = y * w, tol * w.abs()
    if b is not None:
        y = y + b
        tol = tol + U * y.abs()
    return y, tol


def reference(x, block, weight, bias, bw, bb, gate, act, scale, eps, center, kind):
    """total and out of add_norm (x None, weight None: of norm, whose weights are bw and bb) with tolerances."""
    f = lambda t: None if t is None else t.double().cpu()  # noqa: E731
    x, z, weight, bias, bw, bb, gate, scale = (f(t) for t in (x, block, weight, bias, bw, bb, gate, scale))
    tol = torch.zeros_like(z)
    if bw is not None or x is None:
        z, tol = normed(z, tol, bw, bb, center, eps)
    if gate is not None:
        g = {None: lambda t: t, "silu": lambda t: t * torch.sigmoid(t), "sigmoid": torch.sigmoid}[act](gate)
        g = g.view(gate.shape[:-1] + (1,) * (z.dim() - gate.dim()) + gate.shape[-1:])
        z, tol = z * g, tol * g.abs() + 16 * U * (z * g).abs()
    if scale is not None:
        z, tol = z * scale, (tol + U * z.abs()) * scale.abs()
    if x is not None:
        z = z + x
        tol = tol + U * z.abs()
    out = [(z, tol + OUT[kind] * z.abs() + 1e-37)]
    if weight is not None:
        y, ty = normed(z, tol, weight, bias, center, eps)
        out.append((y, ty + OUT[kind] * y.abs() + 1e-37))
    return out


WIDTHS = [1, 2, 3, 7, 8, 9, 31, 32, 42, 64, 100, 256, 384, 509, 1024, 1025, 1500, 2048, 2056, 4096, 4100, 8192, 9001, 20000]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_add_norm_widths(width, kind):
    """One lane's worth to several workgroup's; every operand there and not."""
    note(f"[gpu-test] add_norm {width} {kind}")
    rng = np.random.default_rng(width)
    k = KIND[kind]
    for rows, center in ((1, False), (37, True)):
        x, block, gate = normal(rng, (rows, width), k, 2, 0.5), normal(rng, (rows, width), k, 0.7), normal(rng, (rows, width), k)
        w, bw = normal(rng, (width,), k, 0.2, 1), normal(rng, (width,), k, 0.2, 1)
        b, bb, scale = (normal(rng, (width,), k, 0.3) for _ in range(3))
        eps = 1e-3                                     # rows of one value, less their mean, are zero
        for args in (dict(), dict(block_weight=bw), dict(gate=gate, activation="silu", scale=scale),
                     dict(block_weight=bw, block_bias=bb, gate=gate[0], activation="sigmoid", scale=scale)):
            total, out = ssc.add_norm(x, block, w, b, eps=eps, center=center, **args)
            ref = reference(x, block, w, b, args.get("block_weight"), args.get("block_bias"), args.get("gate"),
                            args.get("activation"), args.get("scale"), eps, center, kind)
            close(total, *ref[0], f"total {sorted(args)}")
            close(out, *ref[1], f"out {sorted(args)}")
        total, out = ssc.add_norm(x, block, gate=gate, scale=scale)
        assert out is None
        close(total, *reference(x, block, None, None, None, None, gate, None, scale, eps, center, kind)[0], "no norm after")
        y = ssc.norm(x, w, b, eps=eps, center=center, gate=gate, activation="silu")
        close(y, *reference(None, x, None, None, w, b, gate, "silu", None, eps, center, kind)[0], "norm")
        y = ssc.norm(x, eps=eps, center=center)
        close(y, *reference(None, x, None, None, None, None, None, None, None, eps, center, kind)[0], "norm alone")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape,lead", [((2, 13, 7, 64), 0), ((2, 13, 7, 64), 1), ((2, 13, 7, 64), 2), ((2, 13, 7, 64), 3),
                                        ((5, 1, 33), 1), ((1, 4, 20), 1), ((70000, 16), 0), ((3, 5, 2500), 1)])
def test_gates_of_images(shape, lead, kind):
    """A gate for every row, for every run of rows and for all."""
    rng = np.random.default_rng(len(shape) * 10 + lead)
    k = KIND[kind]
    x, block, gate = normal(rng, shape, k), normal(rng, shape, k), normal(rng, shape[:lead] + shape[-1:], k)
    w = normal(rng, shape[-1:], k, 0.2, 1)
    total, out = ssc.add_norm(x, block, w, gate=gate, activation="sigmoid")
    ref = reference(x, block, w, None, None, None, gate, "sigmoid", None, 1e-6, False, kind)
    close(total, *ref[0], "total")
    close(out, *ref[1], "out")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width,pad,offset", [(40, 0, 1), (40, 8, 0), (40, 3, 5), (33, 1, 2), (1111, 9, 3), (5000, 7, 1)])
def test_strides_alignment_and_what_is_not_written(width, pad, offset, kind):
    rng = np.random.default_rng(width + pad)
    k, rows = KIND[kind], 41

    def strided():
        flat = normal(rng, (rows * (width + pad) + offset + 64,), k)
        return flat, flat[offset:offset + rows * (width + pad)].view(rows, width + pad)[:, :width]

    (_, x), (_, block), (_, gate), (ft, total), (fo, out) = (strided() for _ in range(5))
    w = normal(rng, (width + 1,), k)[1:]
    before = ft.clone(), fo.clone()
    got = ssc.add_norm(x, block, w, gate=gate, total=total, out=out)
    assert got[0] is total and got[1] is out
    ref = reference(x, block, w, None, None, None, gate, None, None, 1e-6, False, kind)
    close(total, *ref[0], "total")
    close(out, *ref[1], "out")
    for flat, was in zip((ft, fo), before):
        mask = torch.ones_like(flat, dtype=torch.bool)
        mask[offset:offset + rows * (width + pad)].view(rows, width + pad)[:, :width] = False
        assert torch.equal(flat[mask], was[mask])


@pytest.mark.parametrize("width", [40, 9001])
def test_rows_far_apart(width):
    """Rows 2^25 values apart, all within one tensor: the last ones begin behind 2^32 bytes and values."""
    rng = np.random.default_rng(width)
    rows = torch.empty((140, 1 << 25), dtype=torch.bfloat16, device="cuda")
    x, block, gate, total, out = (rows[:, i * width:(i + 1) * width] for i in range(5))
    for t in (x, block, gate):
        t.copy_(normal(rng, (140, width), torch.bfloat16))
    w = normal(rng, (width,), torch.bfloat16, 0.2, 1)
    ssc.add_norm(x, block, w, gate=gate, total=total, out=out)
    ref = reference(x, block, w, None, None, None, gate, None, None, 1e-6, False, "bf16")
    close(total, *ref[0], "total")
    close(out, *ref[1], "out")


def test_more_than_2_to_32_values():
    rows, width = (1 << 32) // 1000 + 77, 1000
    x = torch.randn((rows, width), dtype=torch.bfloat16, device="cuda")
    w = normal(np.random.default_rng(1), (width,), torch.bfloat16, 0.2, 1)
    total, out = ssc.add_norm(x, x, w)
    for s in (slice(0, 50), slice(rows // 2, rows // 2 + 50), slice(rows - 50, rows)):
        ref = reference(x[s], x[s], w, None, None, None, None, None, None, 1e-6, False, "bf16")
        close(total[s], *ref[0], "total")
        close(out[s], *ref[1], "out")


@pytest.mark.parametrize("width", [64, 300, 3000, 20000])
def test_in_place(width):
    """The sum in the residual's or the block's place, the norm in the other's; a gate's."""
    rng = np.random.default_rng(width)
    make = lambda: normal(rng, (19, width), torch.float32)  # noqa: E731
    x, block, gate, w = make(), make(), make(), normal(rng, (width,), torch.float32)
    want = ssc.add_norm(x, block, w, block_weight=w, gate=gate, center=True)
    for which in range(2):
        a, b = x.clone(), block.clone()
        total, out = (a, b) if which == 0 else (b, a)
        ssc.add_norm(a, b, w, block_weight=w, gate=gate, center=True, total=total, out=out)
        assert torch.equal(total, want[0]) and torch.equal(out, want[1])
    y = ssc.norm(x, w, gate=gate)
    a, g = x.clone(), gate.clone()
    assert torch.equal(ssc.norm(a, w, gate=gate, out=a), y) and torch.equal(ssc.norm(x, w, gate=g, out=g), y)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_far_means_and_special_values(kind):
    """A mean a thousand times the spread is taken off first; rows with infinities and
    NaN do not reach other rows; zeros with eps are zeros."""
    rng = np.random.default_rng(5)
    k = KIND[kind]
    x = normal(rng, (50, 96), torch.float32, 1.0, 1000.0).to(k)
    close(ssc.norm(x, center=True), *reference(None, x, None, None, None, None, None, None, None, 1e-6, True, kind)[0], "far")
    x = normal(rng, (9, 96), k)
    clean = ssc.norm(x)
    bad = x.clone()
    bad[3, 5], bad[6, 0] = math.inf, math.nan
    y = ssc.norm(bad)
    keep = [0, 1, 2, 4, 5, 7, 8]
    assert torch.equal(y[keep], clean[keep])
    assert bool(torch.isnan(y[6]).all()) and bool(torch.isnan(y[3, 5])) and float(y[3, :5].abs().max()) == 0.0
    assert torch.equal(ssc.norm(torch.zeros_like(x)), torch.zeros_like(x))
    g = torch.tensor([-math.inf, -200.0, -90.0, 0.0, 90.0, 200.0, math.inf, 1.0], device="cuda").to(k).expand(9, 8).contiguous()
    s = ssc.add_norm(torch.zeros_like(g), torch.ones_like(g), gate=g, activation="sigmoid")[0]
    assert s[0, [0, 1]].tolist() == [0.0, 0.0] and s[0, [3, 4, 5, 6]].tolist() == [0.5, 1.0, 1.0, 1.0]


def test_no_rows_no_work():
    x = torch.empty(0, 24, device="cuda")
    total, out = ssc.add_norm(x, x, torch.ones(24, device="cuda"))
    assert total.shape == out.shape == (0, 24) and ssc.norm(x).shape == (0, 24)


def test_rows_do_not_depend_on_one_another():
    rng = np.random.default_rng(8)
    x, w = normal(rng, (1000, 384), torch.bfloat16), normal(rng, (384,), torch.bfloat16)
    y = ssc.norm(x, w)
    assert torch.equal(ssc.norm(x[777:778], w), y[777:778]) and torch.equal(ssc.norm(x[:500], w), y[:500])


def test_refusals():
    x, w = torch.randn(4, 32, device="cuda"), torch.ones(32, device="cuda")
    for bad in (lambda: ssc.norm(x.cpu()), lambda: ssc.norm(x.half()), lambda: ssc.norm(x, w[:16]), lambda: ssc.norm(x, w.bfloat16()),
                lambda: ssc.norm(x, w, activation="silu"), lambda: ssc.norm(x, w, gate=x, activation="gelu"),
                lambda: ssc.norm(x, w, gate=x[:2]), lambda: ssc.norm(x, w, gate=x[:, :16]), lambda: ssc.norm(x.t(), w),
                lambda: ssc.norm(x, w, out=x[:2]), lambda: ssc.add_norm(x, x[:2], w), lambda: ssc.add_norm(x, x, None, w),
                lambda: ssc.add_norm(x, x, w, block_bias=w), lambda: ssc.add_norm(x, x, w, total=x, out=x),
                lambda: ssc.add_norm(x, x, w, scale=x[:, 0]), lambda: ssc.norm(x[:, :0]),
                lambda: ssc.add_norm(x, x, w, gate=torch.ones(1, 32, device="cuda").expand(4, 32))):
        with pytest.raises(ValueError):
            bad()
    for at in range(4):
        ops = [t.clone().requires_grad_(i == at) for i, t in enumerate((x, x, w, x))]
        with pytest.raises(ValueError, match="gradient"):
            ssc.add_norm(ops[0], ops[1], ops[2], gate=ops[3])
    with pytest.raises(ssc.SscaterError):
        ssc.norm(x, w, eps=-1.0)
