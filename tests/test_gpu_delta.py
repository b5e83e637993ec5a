"""GPU tests of the gated delta rule against the recurrence in 64 bits.

Tolerance (u = 2^-24): with unit keys and 0 <= beta <= 2 the map from one state to the
next does not lengthen a column, so what a token adds to a column's error, in 2-norm, is
carried on times alpha.  A token adds the roundings of its products with the column, of
length key_dim, and, where 64 tokens are taken together, of sums over those: c u (|S| +
|v|) with c = 2 (sqrt(key_dim) + sqrt(64) + 32), the last for the exponentials, norms and
single products.  An output is off by |q| scale times that, by its own sum's 2
(sqrt(key_dim) + 8) u |S| and, stored in bf16, by 2^-8 of itself.
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


def recurrence(S, q, k, v, alpha, beta, scale, kind):
    """One stream in 64 bits: S [heads, dk, dv], q, k [n, heads, dk], v [n, heads, dv], alpha, beta [n, heads]."""
    dk = k.shape[-1]
    c = 2 * (math.sqrt(dk) + 8 + 32) * U
    err = torch.zeros(S.shape[0], S.shape[2], dtype=torch.float64)
    out, tol = torch.empty_like(v), torch.empty_like(v)
    for t in range(v.shape[0]):
        al, be = alpha[t, :, None], beta[t, :, None]
        size = S.norm(dim=1)
        S = al[..., None] * S
        u = be * (v[t] - (S * k[t, :, :, None]).sum(1))
        S = S + k[t, :, :, None] * u[:, None]
        err = al * err + c * (size + S.norm(dim=1) + v[t].abs())
        out[t] = scale * (S * q[t, :, :, None]).sum(1)
        tol[t] = abs(scale) * q[t].norm(dim=-1, keepdim=True) * (err + 2 * (math.sqrt(dk) + 8) * U * S.norm(dim=1))
    return S, err, out, tol + OUT[kind] * out.abs() + 1e-37


def bound(got, ref, tol, what):
    got = got.double().cpu()
    assert got.shape == ref.shape and bool(torch.isfinite(got).all()), what
    worst = float(((got - ref).abs() / tol).max()) if got.numel() else 0.0
    note(f"[gpu-test] {what}: {worst:.3f} of the tolerance")
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


class Case:
    """Tokens of a call as columns of one projection's rows, and the call checked."""

    def __init__(self, seed, counts, heads, qk, dk, dv, kind, raw=True, unit=True, pad=0, hard=False, tail=0):
        rng = self.rng = np.random.default_rng(seed)
        self.counts, self.heads, self.qk, self.dk, self.dv, self.kind = counts, heads, qk, dk, dv, kind
        self.raw, self.unit = raw, unit
        n = sum(counts) + tail
        rows = normal(rng, (n, 2 * qk * dk + heads * dv + 2 * heads + pad), KIND[kind])
        at, parts = pad // 2, []
        for h, d in ((qk, dk), (qk, dk), (heads, dv), (heads, 1), (heads, 1)):
            parts.append(rows[:, at:at + h * d].unflatten(1, (h, d)) if d > 1 else rows[:, at:at + h])
            at += h * d
        self.q, self.k, self.v, self.a, self.b = parts
        if not unit:
            self.k.mul_(0.5 * dk ** -0.5)
        if not raw:
            self.a.copy_(-self.a.float().abs() * (20 if hard else 0.2))
            if hard:
                self.a[torch.from_numpy(rng.random(tuple(self.a.shape)) < 0.05).cuda()] = -math.inf
            self.b.copy_(torch.sigmoid(self.b.float()))
        self.rate = torch.from_numpy(np.exp(rng.uniform(0, math.log(16), heads)).astype(np.float32)).cuda() if raw else None
        self.bias = torch.from_numpy(rng.uniform(-7, -2, heads).astype(np.float32)).cuda() if raw else None
        if raw and hard:
            self.rate, self.bias = self.rate * 20, self.bias + 6
        self.start = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32).cuda()
        self.state = normal(rng, (len(counts), heads, dk, dv), torch.float32, 0.5)
        self.memory = ssc.DeltaMemory(len(counts), heads, dk, dv, qk_heads=qk, dtype=kind, state=self.state.clone())

    def call(self, memory=None, eps=1e-6, **more):
        m = memory or self.memory
        return m.update(self.q, self.k, self.v, self.a, self.b, rate=self.rate, bias=self.bias, eps=eps if self.unit else None,
                        **more)

    def sequences(self):
        """(stream, its tokens' outputs' places, 64-bit results) of every stream."""
        f = lambda t: t.double().cpu()  # noqa: E731
        rep = self.heads // self.qk
        q, k, v, a, b = (f(t) for t in (self.q, self.k, self.v, self.a, self.b))
        if self.unit:
            q, k = (x / torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6) for x in (q, k))
        q, k = q.repeat_interleave(rep, 1), k.repeat_interleave(rep, 1)
        if self.raw:
            x = a + f(self.bias)
            a, b = -f(self.rate) * torch.nn.functional.softplus(x, threshold=40), torch.sigmoid(b)
        at = 0
        for i, n in enumerate(self.counts):
            s = slice(at, at + n)
            at += n
            yield (i, s) + recurrence(f(self.state[i]), q[s], k[s], v[s], torch.exp(a[s]), b[s], self.dk ** -0.5, self.kind)

    def check(self, **more):
        out = self.call(**more)
        assert out.shape == (self.v.shape[0], self.heads, self.dv) and out.dtype == KIND[self.kind]
        for i, s, S, err, ref, tol in self.sequences():
            bound(out[s], ref, tol, f"stream {i} of {self.counts[i]} tokens")
            diff = (self.memory.state[i].double().cpu() - S).norm(dim=1)
            worst = float((diff / (err + 2 * U * S.norm(dim=1) + 1e-37)).max())
            note(f"[gpu-test] state {i}: {worst:.3f} of the tolerance")
            assert worst <= 1.0, f"state {i}: {worst} of the tolerance"
        return out


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dv", [32, 64, 128])
@pytest.mark.parametrize("dk", [32, 64, 128])
def test_sizes_and_lengths(dk, dv, kind):
    """Token by token and over stretches, on either side of a stretch's 64 tokens."""
    for n in (1, 2, 5, 17, 63, 64, 65, 200):
        note(f"[gpu-test] delta {dk} x {dv} {kind}, {n} tokens")
        Case(n + dk, [n, n], 2, 2, dk, dv, kind).check()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("heads,qk", [(1, 1), (3, 1), (6, 2)])
@pytest.mark.parametrize("counts", [[1, 0, 1, 1, 0], [0, 3, 129, 1, 64], [700, 0, 5, 66]])
def test_streams_of_different_lengths(counts, heads, qk, kind):
    """Heads that share keys; streams without tokens keep their state; rows behind the
    last stream are not looked at and left as they were."""
    c = Case(sum(counts) + heads, counts, heads, qk, 64, 32, kind, pad=3, tail=4)
    n = sum(counts)
    for t in (c.q, c.k, c.v, c.a, c.b):
        t[n:] = math.nan
    for limit in (max(counts), None):
        out = torch.full((n + 4, heads, 32), 7.0, dtype=KIND[kind], device="cuda")
        c.memory.state.copy_(c.state)
        got = c.check(start=c.start, max_new=limit, out=out)
        assert got is out and bool((out[n:] == 7.0).all())
        for i, m in enumerate(counts):
            if m == 0:
                assert torch.equal(c.memory.state[i], c.state[i])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("raw,unit,hard", [(False, False, False), (False, True, True), (True, True, True), (True, False, False)])
@pytest.mark.parametrize("n", [3, 150])
def test_gates(n, raw, unit, hard, kind):
    """alpha and beta as they are given (down to alpha = 0) and from a projection's
    columns; keys as they are; heads that forget at once beside others that do not."""
    Case(n, [n], 4, 2, 64, 64, kind, raw=raw, unit=unit, hard=hard).check()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("counts,dk,dv", [([3000, 1500], 32, 32), ([1, 1000, 0, 640], 128, 32), ([2049], 64, 128)])
def test_a_long_stream(counts, dk, dv, kind):
    """Thousands of tokens, one of the heads forgetting hardly anything: streams in
    parts, of which short ones have no second."""
    c = Case(3, counts, 2, 2, dk, dv, kind)
    c.rate[0], c.bias[0] = 0.01, -7.0
    c.check(start=c.start, max_new=max(counts))


def test_parts_of_a_stream_are_the_stream():
    """Tokens in one call or in several give results within each other's tolerance,
    and repeated calls the same bits."""
    c = Case(8, [300], 2, 2, 64, 64, "f32")
    whole = c.call().clone()
    state = c.memory.state.clone()
    c.memory.state.copy_(c.state)
    assert torch.equal(c.call(), whole) and torch.equal(c.memory.state, state)
    c.memory.state.copy_(c.state)
    parts, at = [], 0
    for n in (1, 1, 100, 7, 64, 127):
        s = slice(at, at + n)
        parts.append(c.memory.update(c.q[s], c.k[s], c.v[s], c.a[s], c.b[s], rate=c.rate, bias=c.bias))
        at += n
    (_, _, S, err, ref, tol), = c.sequences()
    bound(torch.cat(parts), ref, tol, "in parts")
    assert bool(((c.memory.state[0].double().cpu() - S).norm(dim=1) <= err + 2 * U * S.norm(dim=1)).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("counts,dk,dv", [([140], 64, 64), ([2, 138], 128, 32), ([5, 4], 32, 64)])
def test_tokens_far_apart(counts, dk, dv, kind):
    """The largest stride, 2^24 elements: a stretch's tokens lie up to 2^32 bytes apart, and the last ones further on."""
    c = Case(sum(counts), counts, 2, 1, dk, dv, kind)
    rows, at = torch.empty((sum(counts), 1 << 24), dtype=KIND[kind], device="cuda"), 1 << 24
    for name in "qkvab":
        t = getattr(c, name)
        width = t[0].numel()
        at -= width
        view = rows[:, at:at + width]
        view.copy_(t.reshape(len(t), -1))
        setattr(c, name, view.unflatten(1, t.shape[1:]) if t.dim() == 3 else view)
    c.check(start=c.start, max_new=max(counts))


def test_more_than_4_gib_of_states():
    """70001 streams of 128 x 128, a token each: the first, the last and one between."""
    n = 70001
    rng = np.random.default_rng(8)
    q, k, v = (normal(rng, (n, 1, 128), torch.float32) for _ in range(3))
    a, b = -normal(rng, (n, 1), torch.float32).abs(), torch.sigmoid(normal(rng, (n, 1), torch.float32))
    state = torch.randn((n, 1, 128, 128), device="cuda")
    pick = [0, 33333, n - 1]
    before = state[pick].double().cpu()
    m = ssc.DeltaMemory(n, 1, 128, 128, state=state)
    out = m.update(q, k, v, a, b)
    q, k, v, a, b = (t[pick].double().cpu()[:, None] for t in (q, k, v, a, b))
    q, k = (x / torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6) for x in (q, k))
    for i, s in enumerate(pick):
        S, err, ref, tol = recurrence(before[i], q[i], k[i], v[i], torch.exp(a[i]), b[i], 128 ** -0.5, "f32")
        bound(out[s:s + 1], ref, tol, f"stream {s}")
        assert bool(((state[s].double().cpu() - S).norm(dim=1) <= err + 2 * U * S.norm(dim=1)).all())


@pytest.mark.parametrize("n", [1, 100, 1500])
def test_initial_states(n):
    """Beginning from other states leaves those as they were and writes the memory's,
    of streams without tokens too; from its own gives the same bits."""
    c = Case(n, [n, 0, n], 2, 1, 32, 64, "f32")
    want = c.call(start=c.start, max_new=n).clone()
    state = c.memory.state.clone()
    first = c.state.clone()
    c.memory.state.fill_(math.nan)
    got = c.call(start=c.start, max_new=n, initial=first)
    assert torch.equal(got, want) and torch.equal(c.memory.state, state) and torch.equal(first, c.state)
    c.memory.state.fill_(5.0)
    none = ssc.DeltaMemory(3, 2, 32, 64, qk_heads=1, state=c.memory.state)
    out = none.update(c.q[:0], c.k[:0], c.v[:0], c.a[:0], c.b[:0])
    assert out.shape == (0, 2, 64) and bool((c.memory.state == 5.0).all())
    none.update(c.q[:0], c.k[:0], c.v[:0], c.a[:0], c.b[:0], initial=first)
    assert torch.equal(c.memory.state, first)
    none.reset()
    assert float(none.state.abs().sum()) == 0.0


@pytest.mark.parametrize("n", [1, 90])
def test_streams_do_not_meet(n):
    """NaN in one stream, head or value column stays there; many streams."""
    c = Case(11, [n] * 300, 2, 2, 32, 32, "bf16")
    want, state = c.call().clone(), None
    state = c.memory.state.clone()
    c.memory.state.copy_(c.state)
    c.v[7 * n, 1, 5] = math.nan
    got = c.call()
    same = torch.ones_like(got, dtype=torch.bool)
    same[7 * n:8 * n, 1, 5] = False
    assert torch.equal(got[same], want[same]) and bool(torch.isnan(got[~same]).all())
    same = torch.ones_like(state, dtype=torch.bool)
    same[7, 1, :, 5] = False
    assert torch.equal(c.memory.state[same], state[same])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["q", "k", "v", "a", "b"])
@pytest.mark.parametrize("at,value", [(70, math.nan), (85, math.inf), (0, -math.inf), (129, math.nan), (700, math.inf)])
def test_no_token_sees_a_later_one(at, value, where, kind):
    """An infinity or NaN in a token reaches none of those before it (nor, in a query,
    those after), and no stream beside it; also where a stream is taken in parts."""
    n = 150 if at < 150 else 1500
    c = Case(15, [n, 90], 2, 1, 64, 32, kind)
    rows = [(i, s, S, err, ref, tol) for i, s, S, err, ref, tol in c.sequences()]
    t = getattr(c, where)
    if where == "v":
        t[at, 1, 3] = value
    elif where in "ab":
        t[at, 1] = value
    else:
        t[at, 0, 5] = value
    out = c.call(start=c.start, max_new=n)
    (_, s0, _, _, ref, tol), (_, s1, S, err, ref1, tol1) = rows
    bound(out[s0][:at], ref[:at], tol[:at], f"before {where}")
    bound(out[s1], ref1, tol1, "the other stream")
    assert bool(((c.memory.state[1].double().cpu() - S).norm(dim=1) <= err + 2 * U * S.norm(dim=1)).all())
    if where == "q":
        bound(out[s0][at + 1:], ref[at + 1:], tol[at + 1:], "after a query")
    elif where == "v":
        assert not bool(torch.isfinite(out[s0][at:, 1, 3]).any())
        out[:, 1, 3] = torch.where(torch.isfinite(out[:, 1, 3]), out[:, 1, 3], ref[0, 0, 0].to(out))
        keep = [i for i in range(32) if i != 3]
        bound(out[s0][:, 1, keep], ref[:, 1, keep], tol[:, 1, keep], "the other values")
    if where in "vab":
        bound(out[s0][:, 0], ref[:, 0], tol[:, 0], "the other head")
    if where == "k":
        assert not bool(torch.isfinite(out[s0][at:]).any())


@pytest.mark.parametrize("what", ["no direction", "large key", "large correction"])
@pytest.mark.parametrize("at", [70, 93, 701])
def test_no_token_sees_what_overflows_later(at, what):
    """Finite tokens whose products are not: a key of zeros taken to unit length without
    an eps, one whose square passes the range, a value whose product with its key does.
    (Without the eps of the 64-bit results a key of length 4 or more is off by 2^-25.)"""
    n = 150 if at < 150 else 1500
    unit = what == "no direction"
    c = Case(16, [n, 90], 2, 1, 64, 32, "f32", raw=False, unit=unit)
    (_, s0, _, _, ref, tol), (_, s1, _, _, ref1, tol1) = c.sequences()
    assert not unit or float(c.k.norm(dim=-1).min()) >= 4
    if unit:
        c.k[at] = 0
    elif what == "large key":
        c.k[at] = 1e25
    else:
        c.k[at] *= 400
        c.v[at, 1, 3] = 1e38
    out = c.call(eps=0.0, start=c.start, max_new=n)
    bound(out[s0][:at], ref[:at], tol[:at], "before")
    bound(out[s1], ref1, tol1, "the other stream")
    if what == "large correction":
        keep = [i for i in range(32) if i != 3]
        assert bool(torch.isfinite(out[s0][:, 1, keep]).all()) and bool(torch.isfinite(out[s0][:, 0]).all())


@pytest.mark.parametrize("n", [1, 130])
def test_a_captured_update_replays(n):
    rng = np.random.default_rng(12)
    c = Case(13, [n, n], 2, 2, 64, 64, "bf16")
    data = [[normal(rng, t.shape, torch.bfloat16) for t in (c.q, c.k, c.v, c.a, c.b)] for _ in range(4)]

    def put(d):
        for t, x in zip((c.q, c.k, c.v, c.a, c.b), d):
            t.copy_(x)

    want = []
    for d in data:
        put(d)
        want.append((c.call().clone(), c.memory.state.clone()))
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        out = c.call()
    torch.cuda.synchronize()
    c.memory.state.copy_(c.state)
    for i, d in enumerate(data):
        put(d)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i][0]) and torch.equal(c.memory.state, want[i][1]), f"replay {i}"
        torch.randn(1000, device="cuda").sum().item()


def test_another_stream():
    c = Case(14, [100, 100], 2, 2, 64, 64, "bf16")
    want = c.call().clone()
    c.memory.state.copy_(c.state)
    s = torch.cuda.Stream()
    got = c.call(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


def test_refusals():
    m = ssc.DeltaMemory(2, 4, 32, 64, qk_heads=2)
    q, v, a = torch.randn(6, 2, 32, device="cuda"), torch.randn(6, 4, 64, device="cuda"), torch.randn(6, 4, device="cuda")
    r = torch.ones(4, device="cuda")
    start = torch.tensor([0, 1, 6], dtype=torch.int32, device="cuda")
    for bad in (lambda: m.update(q[:5], q[:5], v[:5], a[:5], a[:5]), lambda: m.update(q, q[:5], v, a, a),
                lambda: m.update(q.bfloat16(), q, v, a, a), lambda: m.update(q.cpu(), q, v, a, a),
                lambda: m.update(q, q, v[:, :2], a, a), lambda: m.update(q, q, v, a[:, :2], a), lambda: m.update(q[:, 0], q, v, a, a),
                lambda: m.update(q, q, v, a, a, rate=r), lambda: m.update(q, q, v, a, a, rate=r[:2], bias=r[:2]),
                lambda: m.update(q, q, v, a, a, rate=r.bfloat16(), bias=r.bfloat16()),
                lambda: m.update(q, q, v, a, a, start=start.long()), lambda: m.update(q, q, v, a, a, start=start[:2]),
                lambda: m.update(q, q, v, a, a, max_new=2), lambda: m.update(q, q, v, a, a, out=v[:3]),
                lambda: m.update(q, q, v, a, a, initial=m.state[:1]), lambda: m.update(q, q, v.expand(6, 4, 64)[:1].expand(6, 4, 64), a, a),
                lambda: m.update(q.transpose(1, 2).contiguous().transpose(1, 2), q, v, a, a),
                lambda: ssc.DeltaMemory(0, 4, 32, 64), lambda: ssc.DeltaMemory(2, 4, 48, 64), lambda: ssc.DeltaMemory(2, 4, 32, 16),
                lambda: ssc.DeltaMemory(2, 4, 32, 64, qk_heads=3), lambda: ssc.DeltaMemory(2, 4, 32, 64, dtype="f16"),
                lambda: ssc.DeltaMemory(2, 4, 32, 64, state=torch.zeros(2, 4, 64, 32, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    assert float(m.state.abs().sum()) == 0.0
    for at in range(5):
        ops = [t.clone().requires_grad_(i == at) for i, t in enumerate((q, q, v, a, a))]
        with pytest.raises(ValueError, match="gradient"):
            m.update(*ops)
    for more in (dict(eps=-1.0), dict(scale=math.nan), dict(start=start, max_new=7)):
        with pytest.raises(ssc.SscaterError):
            m.update(q, q, v, a, a, **more)
    with pytest.raises(AttributeError):
        m.state = torch.zeros(1)
