"""GPU tests of how near bf16 attention comes to 64 bits, and of infinite values, in
the kernels that take a probability in two bf16 parts.

Tolerance (u = 2^-24): scores are off by 2 (sqrt(D) + 8) u scale sum |q k| and 4 u of
themselves before exp, twice (numerator and sum); sums of n terms by 2 (sqrt(n) + 8) u;
a probability in two bf16 parts by 2^-8 of what the first leaves, itself at most 2^-8 of
the value: 2^-16; all relative to sum p |v|.  Then the output's rounding, half a step of
bf16 or 2^-8 of itself, and 2 u."""
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
BF16 = torch.bfloat16


def normal(rng, shape, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(BF16).cuda()


def reference(q, k, v, seen, part=2.0 ** -16):
    """One sequence, q [n, heads, D], k and v [keys, kv, D], seen [keys] or None: outputs and tolerances."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    if seen is not None:
        k, v = k[seen.cpu()], v[seen.cpu()]
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    group, dim = q.shape[1] // k.shape[1], q.shape[2]
    for h in range(q.shape[1] if len(k) else 0):
        kk, vv, x = k[:, h // group], v[:, h // group], q[:, h]
        s = (x @ kk.t()) / math.sqrt(dim)
        p = torch.softmax(s, -1)
        out[:, h] = p @ vv
        err = 2 * (math.sqrt(dim) + 8) * U * (x.abs() @ kk.abs().t()) / math.sqrt(dim) + 4 * U * s.abs()
        rel = 2 * err.max(-1, keepdim=True).values + 2 * (math.sqrt(len(kk)) + 8) * U + part
        tol[:, h] = rel * (p @ vv.abs()) + (2.0 ** -8 + 2 * U) * out[:, h].abs()
    return out, tol


def close(got, ref, tol, what, where=None):
    got = got.double().cpu()
    where = torch.ones_like(tol, dtype=torch.bool) if where is None else where
    assert bool(torch.isfinite(got[where]).all()), f"{what}: not finite"
    worst = float(((got - ref).abs()[where] / tol.clamp(min=1e-300)[where]).max())
    note(f"[gpu-test] {what}: {worst:.3f} of the tolerance")
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


@pytest.mark.parametrize("rows", [1, 7, 32])
@pytest.mark.parametrize("form", ["rows", "listed", "cache"])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_an_infinite_value_of_few_rows(dim, form, rows):
    """Visible infinities keep their sign in every row, and reach their own column alone."""
    note(f"[gpu-test] infinite values, {rows} rows, {form}, {dim}")
    rng = np.random.default_rng(rows + dim)
    q, k, v = normal(rng, (rows, 2, dim), 2.0), normal(rng, (96, 2, dim)), normal(rng, (96, 2, dim))
    seen = torch.from_numpy(rng.random(96) < 0.7).cuda() if form == "listed" else None
    if seen is not None:
        seen[50] = seen[60] = True
    ref = reference(q, k, v, seen)
    v[50, 0, 3], v[60, 1, 7] = math.inf, -math.inf
    if form == "cache":
        kc, vc = (t.transpose(0, 1).contiguous()[None] for t in (k, v))
        c = ssc.TokenCache(1, 2, dim, 96, dtype="bf16", k=kc, v=vc)
        c.seek([96 - rows])
        out = c.attend(q, 96, causal=False)
    else:
        out = ssc.cross_attend(q, k, v, seen)
    assert bool((out[:, 0, 3] == math.inf).all()) and bool((out[:, 1, 7] == -math.inf).all())
    rest = torch.ones(ref[0].shape, dtype=torch.bool)
    rest[:, 0, 3] = rest[:, 1, 7] = False
    close(out, *ref, "the other values", rest)


@pytest.mark.parametrize("visible", [None, 0.5])
@pytest.mark.parametrize("queries,group,keys", [(33, 1, 700), (64, 1, 64), (20, 3, 1500), (65, 1, 4096), (130, 2, 333), (300, 1, 9001)])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_many_bf16_rows_are_off_by_the_rounding_of_the_output_alone(dim, queries, group, keys, visible):
    """More than 32 rows of a key head, up to 64 and more; rounded=True: a probability is off by 2^-8."""
    note(f"[gpu-test] cross {queries} x {group} rows, {keys} keys of {dim}, visible {visible}")
    rng = np.random.default_rng(keys + dim)
    q, k, v = normal(rng, (queries, 2 * group, dim), 2.0), normal(rng, (keys, 2, dim)), normal(rng, (keys, 2, dim))
    seen = None if visible is None else torch.from_numpy(rng.random(keys) < visible).cuda()
    close(ssc.cross_attend(q, k, v, seen), *reference(q, k, v, seen), "two parts")
    close(ssc.cross_attend(q, k, v, seen, rounded=True), *reference(q, k, v, seen, 2.0 ** -8), "rounded")


@pytest.mark.parametrize("rounded", [False, True])
@pytest.mark.parametrize("rows", [33, 64, 130])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_an_infinite_value_of_many_rows(dim, rows, rounded):
    note(f"[gpu-test] infinite values, {rows} rows of {dim}, rounded {rounded}")
    rng = np.random.default_rng(rows + dim)
    q, k, v = normal(rng, (rows, 2, dim), 2.0), normal(rng, (192, 2, dim)), normal(rng, (192, 2, dim))
    ref = reference(q, k, v, None, 2.0 ** -8 if rounded else 2.0 ** -16)
    v[50, 0, 3], v[60, 1, 7] = math.inf, -math.inf
    out = ssc.cross_attend(q, k, v, rounded=rounded)
    assert bool((out[:, 0, 3] == math.inf).all()) and bool((out[:, 1, 7] == -math.inf).all())
    rest = torch.ones(ref[0].shape, dtype=torch.bool)
    rest[:, 0, 3] = rest[:, 1, 7] = False
    close(out, *ref, "the other values", rest)


def test_where_nothing_is_rounded():
    """float32, and up to 32 rows: the same bits either way."""
    rng = np.random.default_rng(3)
    for kind, queries in ((torch.float32, 100), (torch.float32, 5), (BF16, 32), (BF16, 1)):
        q, k, v = (normal(rng, (n, 2, 64)).to(kind) for n in (queries, 500, 500))
        assert torch.equal(ssc.cross_attend(q, k, v), ssc.cross_attend(q, k, v, rounded=True))
