"""GPU tests of cross_attend against a plain implementation in 64 bits.

Tolerances as for the attention over the token cache (u = 2^-24): scores are off by
2 (sqrt(D) + 8) u scale sum |q k| and by 2 u of themselves before exp, a sum over n keys
by 2 (sqrt(n) + 8) u, in bf16 a probability by 2^-8 (half a step is 2^-9, in the product
and in what it is compared with), all relative to sum p |v|; the output by u, in bf16
2^-8, of itself.
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


def normal(rng, shape, kind, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(kind).cuda()


def reference(q, k, v, seen, scale, kind):
    """One sequence: q [n, heads, D], k and v [keys, kv, D], seen [keys] or None."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    if seen is not None:
        k, v = k[seen.bool().cpu()], v[seen.bool().cpu()]
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    if k.shape[0] == 0:
        return out, tol
    group, dim = q.shape[1] // k.shape[1], q.shape[2]
    for h in range(q.shape[1]):
        kk, vv, x = k[:, h // group], v[:, h // group], q[:, h]
        s = scale * (x @ kk.t())
        p = torch.softmax(s, -1)
        out[:, h] = p @ vv
        err = 2 * (math.sqrt(dim) + 8) * U * abs(scale) * (x.abs() @ kk.abs().t()) + 4 * U * s.abs()
        rel = 2 * err.max(-1, keepdim=True).values + 2 * (math.sqrt(k.shape[0]) + 8) * U + (2.0 ** -8 if kind == "bf16" else 0)
        tol[:, h] = rel * (p @ vv.abs()) + OUT[kind] * out[:, h].abs()
    return out, tol


def close(got, ref, tol, what):
    got = got.double().cpu()
    assert got.shape == ref.shape
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    none = tol == 0
    assert float(got[none].abs().sum()) == 0.0, f"{what}: a row without keys is not zero"
    worst = float(((got - ref).abs()[~none] / tol[~none]).max()) if bool((~none).any()) else 0.0
    note(f"[gpu-test] {what}: {worst:.3f} of the tolerance")
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


def check(rng, batch, queries, keys, heads, kv, dim, kind, visible=None, scale=None, mask_kind=torch.bool, std=2.0):
    note(f"[gpu-test] cross {batch} x {queries} to {keys}, {heads}/{kv} x {dim} {kind} visible {visible}")
    q = normal(rng, (batch, queries, heads, dim), KIND[kind], std)
    kv_rows = normal(rng, (batch, keys, 2, kv, dim), KIND[kind])
    k, v, mask = kv_rows[:, :, 0], kv_rows[:, :, 1], None
    if visible is not None:
        mask = torch.from_numpy(rng.random((batch, keys)) < visible).cuda()
        mask = mask if mask_kind is torch.bool else mask.to(torch.uint8) * 200
        # what is not visible does not matter
        junk = torch.tensor([math.nan, math.inf, -math.inf, 3e38], device="cuda").to(KIND[kind])
        hidden = ~mask.bool()
        kv_rows[hidden] = junk[torch.randint(0, 4, (int(hidden.sum()), 1, 1, 1), device="cuda")].expand(-1, 2, kv, dim)
    out = ssc.cross_attend(q, k, v, mask, scale=scale)
    assert out.shape == q.shape
    for b in range(batch):
        ref = reference(q[b], k[b], v[b], None if mask is None else mask[b], dim ** -0.5 if scale is None else scale, kind)
        close(out[b], *ref, f"sequence {b}")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("queries,group", [(1, 1), (3, 4), (33, 1), (20, 3), (65, 1), (130, 2)])
@pytest.mark.parametrize("visible", [None, 0.3])
def test_forms(queries, group, dim, kind, visible):
    """Every kernel (up to 32 rows of a key head, up to 64, more) over keys that end
    inside a tile, as they lie and listed."""
    rng = np.random.default_rng(queries * 100 + dim + group)
    for keys in (1, 31, 64, 700):
        check(rng, 2, queries, keys, 2 * group, 2, dim, kind, visible)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("queries,keys,visible", [(1, 40000, None), (5, 33333, 0.1), (300, 5000, None), (200, 70000, 0.02),
                                                  (40, 16385, 0.5), (1, 16384, 0.999), (40, 50000, 0.0), (1, 16389, 0.0)])
def test_long_and_listed(queries, keys, visible, kind):
    """Keys split over workgroups; lists of several workgroups; lists without an entry."""
    check(np.random.default_rng(keys), 1, queries, keys, 2, 1, 64, kind, visible, mask_kind=torch.uint8)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dim,heads,kv", [(32, 8, 8), (64, 4, 1), (128, 6, 3)])
def test_sequences_of_different_lengths(dim, heads, kv, masked, kind):
    """Sequences without queries, without keys, with every key hidden; rows behind the
    last sequence, of queries, keys and mask, are not looked at and left as they were."""
    rng = np.random.default_rng(dim + masked)
    for nq, nk in (([3, 0, 70, 1, 9], [500, 40, 0, 1, 2222]), ([1, 2, 1, 0, 1], [4000, 100, 0, 77, 90000])):
        tail = 6
        total_q, total_k = sum(nq) + tail, sum(nk) + tail
        q, k, v = (normal(rng, (n, h, dim), KIND[kind]) for n, h in ((total_q, heads), (total_k, kv), (total_k, kv)))
        mask = torch.from_numpy(rng.random(total_k) < 0.4).cuda() if masked else None
        if masked:
            mask[sum(nk[:4]):sum(nk)] = masked and nk[4] == 90000
            mask[sum(nk):] = True
        for t in (q[sum(nq):], k[sum(nk):], v[sum(nk):]):
            t.fill_(math.nan)
        starts = [torch.tensor([0] + list(np.cumsum(n)), dtype=torch.int32).cuda() for n in (nq, nk)]
        out = torch.full_like(q, 7.0)
        for limits in (dict(max_q=max(nq), max_k=max(nk)), {}):
            got = ssc.cross_attend(q, k, v, mask, *starts, out=out, **limits)
            assert got is out and bool((out[sum(nq):] == 7.0).all())
            a = c = 0
            for b, (n, m) in enumerate(zip(nq, nk)):
                ref = reference(q[a:a + n], k[c:c + m], v[c:c + m], None if mask is None else mask[c:c + m], dim ** -0.5, kind)
                close(out[a:a + n], *ref, f"sequence {b}")
                a, c = a + n, c + m


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("queries", [2, 50, 100])
def test_strides_and_the_axis_that_may_be_missing(queries, kind):
    """Queries, keys and values as columns of wider rows; one sequence of three axes."""
    rng = np.random.default_rng(queries)
    rows = normal(rng, (queries, 4 * 32 + 32), KIND[kind])
    cells = normal(rng, (333, 5 * 64), KIND[kind])
    q, k, v = rows[:, 16:144].unflatten(1, (4, 32)), cells[:, 64:128].unflatten(1, (2, 32)), cells[:, 192:256].unflatten(1, (2, 32))
    close(ssc.cross_attend(q, k, v), *reference(q, k, v, None, 32 ** -0.5, kind), "columns")
    k, v = normal(rng, (90, 2, 32), KIND[kind]), cells[:90, 192:256].unflatten(1, (2, 32))
    close(ssc.cross_attend(q, k, v), *reference(q, k, v, None, 32 ** -0.5, kind), "keys and values of different strides")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [32, 128])
@pytest.mark.parametrize("queries,masked", [(1, False), (2, True), (50, False), (140, True), (130, False)])
def test_rows_far_apart(queries, masked, dim, kind):
    """The largest stride, 2^24 elements: a tile's rows lie up to 2^32 bytes apart, and the last ones further on."""
    note(f"[gpu-test] cross {queries} queries, rows 2^24 elements apart, {dim} {kind}")
    rng = np.random.default_rng(queries)
    rows = torch.empty((140, 1 << 24), dtype=KIND[kind], device="cuda")
    rows[:, -6 * dim:] = normal(rng, (140, 6 * dim), KIND[kind])
    q, k, v = (rows[:, (i - 6) * dim:(i - 4) * dim or None].unflatten(1, (2, dim)) for i in (0, 2, 4))
    mask = torch.from_numpy(rng.random(140) < 0.6).cuda() if masked else None
    close(ssc.cross_attend(q[:queries], k, v, mask), *reference(q[:queries], k, v, mask, dim ** -0.5, kind), "far apart")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("queries", [1, 40, 200])
def test_scales_and_large_scores(queries, kind):
    rng = np.random.default_rng(queries)
    for scale in (0.0, -0.3, 1e-35, 2.0):
        check(rng, 1, queries, 300, 2, 2, 32, kind, 0.5, scale=scale, std=1.0)
    check(rng, 1, queries, 300, 2, 2, 64, kind, None, std=40.0)


@pytest.mark.parametrize("queries", [1, 40, 200])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_infinities_that_are_seen(queries, kind):
    """Visible infinities and NaN go where the formula takes them, to their own head's
    columns and no further."""
    rng = np.random.default_rng(9)
    q, k, v = (normal(rng, (n, 2, 32), KIND[kind]) for n in (queries, 100, 100))
    clean = ssc.cross_attend(q, k, v)
    v[50, 0, 3], v[60, 1, 7] = math.inf, math.nan
    out = ssc.cross_attend(q, k, v)
    assert bool((out[:, 0, 3] == math.inf).all()) and bool(torch.isnan(out[:, 1, 7]).all())
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[:, 0, 3] = rest[:, 1, 7] = False
    ref = reference(q, k, v.nan_to_num(0, 0, 0), None, 32 ** -0.5, kind)
    got = torch.where(rest, out, clean)
    ok = rest.cpu()
    assert bool(((got.double().cpu() - ref[0]).abs()[ok] <= ref[1][ok]).all())
    k[10] = -math.inf * q[0].sign()                    # a score of minus infinity for the first query
    v.nan_to_num_(0, 0, 0)
    one = ssc.cross_attend(q[:1], k, v)
    hidden = torch.ones(100, dtype=torch.bool, device="cuda")
    hidden[10] = False
    close(one, *reference(q[:1], k, v, hidden, 32 ** -0.5, kind), "minus infinity")
    every = torch.full_like(k[:5], -math.inf)
    assert bool(torch.isnan(ssc.cross_attend(q.abs() + 1, every, v[:5])).all())


def test_bits_depend_on_the_inputs_alone():
    """The same call twice, after other kernels and with other batches' sequences."""
    rng = np.random.default_rng(4)
    q, k, v = (normal(rng, (2, n, 2, 64), torch.bfloat16) for n in (100, 5000, 5000))
    mask = torch.from_numpy(rng.random((2, 5000)) < 0.2).cuda()
    want = ssc.cross_attend(q, k, v, mask)
    for _ in range(3):
        ssc.linear(torch.randn(3000, 512, device="cuda"), torch.randn(512, 512, device="cuda"))
        assert torch.equal(ssc.cross_attend(q, k, v, mask), want)
    other = q.clone()
    other[1] *= 3
    assert torch.equal(ssc.cross_attend(other, k, v, mask)[0], want[0])
    listed = mask[0].nonzero().flatten()
    alone = ssc.cross_attend(q[0], k[0][listed].contiguous(), v[0][listed].contiguous())
    ref = reference(q[0], k[0], v[0], mask[0], 64 ** -0.5, "bf16")
    close(alone, *ref, "gathered by the caller")


def test_many_sequences():
    """More sequences than a grid has rows of workgroups, of one key each: its value p v /
    p, three roundings (the product, the reciprocal, which may be a whole step off, and
    the product with it) or 4 u."""
    rng = np.random.default_rng(6)
    batch = 70001
    q, k, v = (normal(rng, (batch, 1, 1, 32), torch.float32) for _ in range(3))
    mask = torch.from_numpy(rng.random((batch, 1)) < 0.5).cuda()
    out = ssc.cross_attend(q, k, v, mask)
    ref = torch.where(mask[:, :, None, None], v, torch.zeros_like(v)).double()
    assert bool(((out.double() - ref).abs() <= 4 * U * ref.abs()).all())


def test_a_captured_call_replays():
    rng = np.random.default_rng(7)
    q, k, v = (torch.empty(1, n, 4, 32, device="cuda") for n in (60, 4000, 4000))
    mask = torch.empty(1, 4000, dtype=torch.bool, device="cuda")
    data = [[normal(rng, t.shape, torch.float32) for t in (q, k, v)] + [torch.from_numpy(rng.random((1, 4000)) < p).cuda()]
            for p in (0.5, 0.0, 0.01, 1.0)]
    for t, x in zip((q, k, v, mask), data[0]):
        t.copy_(x)
    want = [ssc.cross_attend(*d) for d in data]
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        out = ssc.cross_attend(q, k, v, mask)
    for i in (0, 1, 2, 3, 1, 0):
        for t, x in zip((q, k, v, mask), data[i]):
            t.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i]), f"replay {i}"
        torch.randn(1000, device="cuda").sum().item()


def test_another_stream():
    rng = np.random.default_rng(10)
    q, k, v = (normal(rng, (2, n, 2, 64), torch.bfloat16) for n in (10, 3000, 3000))
    mask = torch.from_numpy(rng.random((2, 3000)) < 0.2).cuda()
    want = ssc.cross_attend(q, k, v, mask)
    s = torch.cuda.Stream()
    got = ssc.cross_attend(q, k, v, mask, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


def test_refusals():
    q, k = torch.randn(2, 3, 4, 32, device="cuda"), torch.randn(2, 9, 2, 32, device="cuda")
    start = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
    mask = torch.ones(2, 9, dtype=torch.bool, device="cuda")
    for bad in (lambda: ssc.cross_attend(q.cpu(), k, k), lambda: ssc.cross_attend(q.half(), k, k),
                lambda: ssc.cross_attend(q, k.bfloat16(), k), lambda: ssc.cross_attend(q, k, k[:, :8]),
                lambda: ssc.cross_attend(q, k[:1], k[:1]), lambda: ssc.cross_attend(q[:, :, :3], k, k),
                lambda: ssc.cross_attend(q, k, k, mask.float()), lambda: ssc.cross_attend(q, k, k, mask[:, :8]),
                lambda: ssc.cross_attend(q, k, k, mask[:1]), lambda: ssc.cross_attend(q, k, k, q_start=start, k_start=start),
                lambda: ssc.cross_attend(q[0], k[0], k[0], q_start=start), lambda: ssc.cross_attend(q, k, k, max_q=3),
                lambda: ssc.cross_attend(q[0], k[0], k[0], q_start=start.long(), k_start=start.long()),
                lambda: ssc.cross_attend(q[0], k[0], k[0], q_start=start, k_start=start[:2]),
                lambda: ssc.cross_attend(q[..., :16], k[..., :16], k[..., :16]), lambda: ssc.cross_attend(q, k, k, out=q[:1]),
                lambda: ssc.cross_attend(q[..., 1:], k[..., 1:], k[..., 1:]), lambda: ssc.cross_attend(q[0, 0], k[0, 0], k[0, 0]),
                lambda: ssc.cross_attend(q, k.transpose(1, 2), k.transpose(1, 2)),
                lambda: ssc.cross_attend(q, torch.randn(2 * 9 * 66 + 1, device="cuda")[1:].view(2, 9, 66)[..., :64].unflatten(2, (2, 32)), k)):
        with pytest.raises(ValueError):
            bad()
    for at in range(3):
        ops = [t.clone().requires_grad_(i == at) for i, t in enumerate((q, k, k))]
        with pytest.raises(ValueError, match="gradient"):
            ssc.cross_attend(*ops)
    with pytest.raises(ssc.SscaterError):
        ssc.cross_attend(q, k, k, scale=math.nan)
    assert ssc.cross_attend(q[:, :0], k, k).shape == (2, 0, 4, 32)
    assert float(ssc.cross_attend(q, k[:, :0], k[:, :0]).abs().sum()) == 0.0
    assert float(ssc.cross_attend(q, k[:, :0], k[:, :0], mask[:, :0]).abs().sum()) == 0.0
