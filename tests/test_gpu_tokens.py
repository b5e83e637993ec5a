"""GPU tests of the token operators against plain implementations in 64 bits.

Tolerances, from the arithmetic (u = 2^-24 for fp32, o = 2^-8 the rounding of a
bf16 output, none for fp32):
  linear  a sum of K fp32 products in fp32, its errors about sqrt(K) u of the
          sum A of the absolute products (8 more roundings for the parts and the
          epilogue): 2 (sqrt(K) + 8) u A, times the largest slope 1.13 of an
          activation, 4 u |z| for its own error, then u and o of the result
  append  a norm over D values, two products and a turn: 16 u of the pair's
          size, 2 pi 2^-25 radians for the angle in turns, then o
  attend  scores: 2 (sqrt(D) + 8) u scale sum |q k| and 2 u of themselves before
          exp; probabilities' sums 2 (sqrt(n) + 8) u; in bf16 o for every
          probability; all relative to sum p |v|, then u and o of the result
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


def close(got, ref, tol, what):
    got = got.double().cpu()
    assert got.shape == ref.shape
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN elsewhere"
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), f"{what}: infinities"
    ok = ~(inf | torch.isnan(ref))
    worst = float(((got - ref).abs()[ok] / tol[ok].clamp(min=1e-300)).max()) if bool(ok.any()) else 0.0
    note(f"[gpu-test] {what}: {worst:.3f} of the tolerance")
    assert worst <= 1.0, f"{what}: {worst} of the tolerance"


# ---- linear ---------------------------------------------------------------------------------
def linear_ref(x, w, b, act, r, kind):
    x, w = x.double().cpu(), w.double().cpu()
    z = x @ w.t()
    size = x.abs().nan_to_num(0, 0, 0) @ w.abs().nan_to_num(0, 0, 0).t()
    if b is not None:
        z, size = z + b.double().cpu(), size + b.double().cpu().abs()
    y = {"none": z, "relu": torch.where(z < 0, 0 * z.clamp(min=-1), z), "silu": z * torch.sigmoid(z),
         "gelu": 0.5 * z * torch.special.erfc(-z / math.sqrt(2))}[act]
    tol = 1.13 * 2 * (math.sqrt(x.shape[-1]) + 8) * U * size + 4 * U * z.abs() + 1e-37
    if r is not None:
        y = y + r.double().cpu()
        tol = tol + U * y.abs()
    return y, tol + OUT[kind] * y.abs()


SHAPES = [(1, 1, 1), (1, 9, 64), (3, 17, 5), (4, 256, 1024), (16, 256, 42), (17, 8, 16), (33, 64, 16), (65, 72, 33),
          (127, 129, 127), (129, 128, 128), (200, 1000, 300), (2050, 384, 42), (5, 2048, 33), (64, 1536, 96),
          (300, 96, 513), (1000, 16, 16), (4100, 40, 260)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_linear_shapes(rows, cin, cout, kind):
    note(f"[gpu-test] linear {rows} {cin} {cout} {kind}")
    rng = np.random.default_rng(rows * 7919 + cin * 31 + cout)
    x, w = normal(rng, (rows, cin), KIND[kind]), normal(rng, (cout, cin), KIND[kind], cin ** -0.5)
    b, r = normal(rng, (cout,), KIND[kind]), normal(rng, (rows, cout), KIND[kind])
    for act, bias, res in (("none", None, None), ("relu", b, None), ("gelu", b, r), ("silu", None, r)):
        y = ssc.linear(x, w, bias, activation=act, residual=res)
        close(y, *linear_ref(x, w, bias, act, res, kind), f"{act}")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", [(33000, 72, 500), (32800, 200, 512), (16500, 8, 1024), (33024, 64, 512),
                                           (20000, 24, 64), (17000, 16, 42), (16385, 33, 7)])
def test_linear_many_rows(rows, cin, cout, kind):
    """Several tiles for every workgroup, with ragged edges, one to four steps of K."""
    note(f"[gpu-test] linear {rows} {cin} {cout} {kind}")
    rng = np.random.default_rng(rows + cin + cout)
    x, w = normal(rng, (rows, cin), KIND[kind]), normal(rng, (cout, cin), KIND[kind], cin ** -0.5)
    b, r = normal(rng, (cout,), KIND[kind]), normal(rng, (rows, cout), KIND[kind])
    for act, bias, res in (("gelu", b, None), ("none", None, r)):
        close(ssc.linear(x, w, bias, activation=act, residual=res), *linear_ref(x, w, bias, act, res, kind), act)


@pytest.mark.parametrize("rows,cin,cout", [(65000, 72, 500), (60000, 200, 384), (27500, 8, 130), (65024, 64, 512),
                                           (27000, 136, 128)])
def test_linear_over_full_passes(rows, cin, cout):
    """Sizes whose tiles of 256 x 128 fill the card once or several times, ragged
    and whole, one to four steps of K."""
    note(f"[gpu-test] linear {rows} {cin} {cout}")
    rng = np.random.default_rng(rows + cin + cout)
    x, w = normal(rng, (rows, cin), torch.bfloat16), normal(rng, (cout, cin), torch.bfloat16, cin ** -0.5)
    b, r = normal(rng, (cout,), torch.bfloat16), normal(rng, (rows, cout), torch.bfloat16)
    for act, bias, res in (("gelu", b, None), ("none", None, r)):
        close(ssc.linear(x, w, bias, activation=act, residual=res), *linear_ref(x, w, bias, act, res, "bf16"), act)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (8, 0), (8, 8), (3, 5), (64, 0)])
def test_linear_strides_and_alignment(kind, pad, offset):
    """Rows further apart than they are long, starting off a boundary; nothing
    outside the output's rows is written."""
    rng = np.random.default_rng(pad * 100 + offset)
    rows, cin, cout = 150, 200, 72

    def strided(n, width):
        flat = normal(rng, (n * (width + pad) + offset,), KIND[kind])
        return flat, flat[offset:].view(n, width + pad)[:, :width]

    (_, x), (_, w), (_, r), (flat, out) = strided(rows, cin), strided(cout, cin), strided(rows, cout), strided(rows, cout)
    before = flat.clone()
    y = ssc.linear(x, w, activation="relu", residual=r, out=out)
    assert y is out
    close(y, *linear_ref(x, w, None, "relu", r, kind), f"pad {pad} offset {offset}")
    mask = torch.ones_like(flat, dtype=torch.bool)
    mask[offset:].view(rows, cout + pad)[:, :cout] = False
    assert torch.equal(flat[mask], before[mask])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_linear_over_maps_and_in_place(kind):
    """A 1x1 head over a [batch, H, W, C] map; the residual as the output."""
    rng = np.random.default_rng(3)
    x, w, b = normal(rng, (2, 13, 7, 64), KIND[kind]), normal(rng, (42, 64), KIND[kind], 0.1), normal(rng, (42,), KIND[kind])
    y = ssc.linear(x, w, b)
    assert y.shape == (2, 13, 7, 42)
    ref, tol = linear_ref(x.view(-1, 64), w, b, "none", None, kind)
    close(y.view(-1, 42), ref, tol, "map")
    r = normal(rng, (2, 13, 7, 42), KIND[kind])
    ref, tol = linear_ref(x.view(-1, 64), w, b, "gelu", r.view(-1, 42), kind)
    assert ssc.linear(x, w, b, activation="gelu", residual=r, out=r) is r
    close(r.view(-1, 42), ref, tol, "in place")
    assert ssc.linear(x[:, :0], w, b).shape == (2, 0, 7, 42)


def test_linear_f32_holds_24_bits():
    """Channels 2^30 apart with weights the other way round, and values near
    the largest: every product counts with its 24 bits."""
    rng = np.random.default_rng(11)
    n = 64
    scale = torch.from_numpy(2.0 ** rng.integers(-15, 16, n)).float().cuda()
    x, w = normal(rng, (100, n), torch.float32) * scale, normal(rng, (64, n), torch.float32) / scale
    close(ssc.linear(x, w), *linear_ref(x, w, None, "none", None, "f32"), "far apart")
    x, w = torch.full((3, 1), 3.4e38, device="cuda"), torch.full((5, 1), 1.0, device="cuda")
    assert torch.equal(ssc.linear(x, w), torch.full((3, 5), 3.4e38, device="cuda"))


@pytest.mark.parametrize("rows", [4, 40, 300])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_linear_infinities_and_nan(kind, rows):
    """They reach the outputs of their own row or channel, as the formula has it."""
    rng = np.random.default_rng(5)
    x, w = normal(rng, (rows, 72), KIND[kind]), normal(rng, (48, 72), KIND[kind])
    x[1, 3], x[2, 70], x[3, 0] = math.inf, math.nan, -math.inf
    w[7, 9] = math.inf
    b = normal(rng, (48,), KIND[kind])
    for act in ("none", "relu"):
        close(ssc.linear(x, w, b, activation=act), *linear_ref(x, w, b, act, None, kind), f"special {act} {rows}")


def test_linear_rows_beyond_32_bits():
    """Rows whose offsets pass 2^31 elements."""
    rows, ld = 1040, (1 << 21) + 8
    flat = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(6)
    data = normal(rng, (rows, 64), torch.bfloat16)
    x = flat.view(rows, ld)[:, :64]
    x.copy_(data)
    w = normal(rng, (24, 64), torch.bfloat16)
    out = flat.view(rows, ld)[:, 64:88]
    ssc.linear(x, w, out=out)
    close(out, *linear_ref(data, w, None, "none", None, "bf16"), "far rows")


# ---- the cache and its attention ---------------------------------------------------------------
class Streams:
    """A plain model of the token streams: everything they ever saw, on the CPU."""

    def __init__(self, rng, batch, kv, dim, sinks, capacity, kind, past=0):
        self.rng, self.kind, self.kv, self.dim = rng, kind, kv, dim
        self.cache = ssc.TokenCache(batch, kv, dim, capacity, sinks=sinks, dtype=kind)
        self.cache.k.fill_(math.nan)          # slots that no token was put into are never read
        self.cache.v.fill_(math.nan)
        self.past = [past] * batch if isinstance(past, int) else list(past)
        self.base = list(self.past)           # positions before these were never held
        self.k = [torch.zeros(0, kv, dim, dtype=torch.float64) for _ in range(batch)]
        self.v = [torch.zeros(0, kv, dim, dtype=torch.float64) for _ in range(batch)]
        if any(self.past):
            self.cache.seek(self.past)

    def slot(self, j):
        c = self.cache
        return j if j < c.sinks else c.sinks + (j - c.sinks) % (c.capacity - c.sinks)


def turn(x, weight, pos, inv_freq, sections, even, eps):
    """[T, heads, D] in 64 bits, and the pairs' sizes."""
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight if weight is not None else x
    dim = x.shape[-1]
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    t = pos.double()[:, axis] * inv_freq.double()
    c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
    a, b = (x[..., 0::2], x[..., 1::2]) if even else (x[..., :dim // 2], x[..., dim // 2:])
    size = torch.sqrt(a * a + b * b)
    a, b = a * c - b * s, a * s + b * c
    join = (lambda p, q: torch.stack([p, q], -1).flatten(-2)) if even else (lambda p, q: torch.cat([p, q], -1))
    return join(a, b), join(size, size)


def attend_ref(q, k, v, p, last, low, sinks, scale, kind, base):
    """One sequence: q [n, heads, D], k and v [positions from base, kv, D]."""
    n, heads, dim = q.shape
    group = heads // k.shape[1]
    j = torch.arange(base, base + k.shape[0])
    out, tol = torch.empty_like(q), torch.empty_like(q)
    for i in range(n):
        seen = (j <= last[i]) & ((j >= low[i]) | (j < sinks))
        for h in range(heads):
            kk, vv = k[seen, h // group], v[seen, h // group]
            s = scale * (kk @ q[i, h])
            pr = torch.softmax(s, 0)
            out[i, h] = pr @ vv
            err = 2 * (math.sqrt(dim) + 8) * U * scale * (kk.abs() @ q[i, h].abs()) + 4 * U * s.abs()
            rel = 2 * float(err.max()) + 2 * (math.sqrt(len(s)) + 8) * U + (2.0 ** -8 if kind == "bf16" else 0)
            tol[i, h] = rel * (pr @ vv.abs()) + OUT[kind] * out[i, h].abs()
    return out, tol


def run_call(st, new, heads, window, causal, even=False, norm=True, sections=None, ragged=None, stream=None, pad=0):
    """One append, attend and advance, each checked."""
    c, rng, kind = st.cache, st.rng, st.kind
    counts = ragged if ragged is not None else [new] * c.batch
    total = sum(counts)
    start = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32).cuda() if ragged is not None else None
    most = max(counts) if ragged is not None else None
    sections = sections or (st.dim // 4, st.dim // 8, st.dim // 8)
    rot = ssc.Rotary(None, sections, interleaved=even)
    width = (heads + 2 * st.kv) * st.dim
    qkv = normal(rng, (total, width + pad), KIND[kind])[:, :width]
    pos = torch.from_numpy(rng.integers(-5, 3000000, (total, len(sections))).astype(np.int32)).cuda()
    qw, kw = (normal(rng, (st.dim,), KIND[kind]) * 0.2 + 1 for _ in range(2)) if norm else (None, None)
    q = c.append(qkv, pos, rot, heads, q_weight=qw, k_weight=kw, start=start, max_new=most, stream=stream)
    out = c.attend(q, window, start=start, max_new=most, causal=causal, stream=stream)
    c.advance(total, start=start, max_new=most, stream=stream)
    torch.cuda.synchronize()
    x = qkv.double().cpu().view(total, heads + 2 * st.kv, st.dim)
    cpu = lambda t: None if t is None else t.double().cpu()  # noqa: E731
    args = (pos.cpu(), rot.inv_freq.cpu(), sections, even, 1e-6)
    rq, sq = turn(x[:, :heads], cpu(qw), *args)
    rk, sk = turn(x[:, heads:heads + st.kv], cpu(kw), *args)
    slack = 16 * U + 2 * math.pi * 2.0 ** -25
    close(q, rq, slack * sq + OUT[kind] * rq.abs(), "queries")
    row = 0
    ck, cv = c.k.double().cpu(), c.v.double().cpu()
    for b, n in enumerate(counts):
        past = st.past[b]
        at = [st.slot(past + i) for i in range(n)]
        keep = [i for i in range(n) if at[i] not in at[i + 1:]]
        if keep:
            rows = torch.tensor(keep) + row
            slots = torch.tensor([at[i] for i in keep])
            close(ck[b][:, slots].transpose(0, 1), rk[rows], slack * sk[rows] + OUT[kind] * rk[rows].abs(), "keys")
            assert torch.equal(cv[b][:, slots].transpose(0, 1), x[rows, heads + st.kv:])
        # the streams as the cache has them, so that attention is checked by itself
        st.k[b] = torch.cat([st.k[b], torch.empty(n, st.kv, st.dim, dtype=torch.float64)])
        st.v[b] = torch.cat([st.v[b], x[row:row + n, heads + st.kv:]])
        for i in keep:
            st.k[b][past - st.base[b] + i] = ck[b][:, at[i]]
        p = [past + i for i in range(n)]
        last = p if causal else [past + n - 1] * n
        low = [(t if causal else past) - window + 1 for t in p]
        # positions that this stream never held are not asked for
        assert n == 0 or st.base[b] == 0 or low[0] >= st.base[b] and c.sinks == 0
        ref, tol = attend_ref(q[row:row + n].double().cpu(), st.k[b], st.v[b], p, last, low, c.sinks,
                              st.dim ** -0.5, kind, st.base[b])
        close(out[row:row + n], ref, tol, f"attend b {b} past {past} new {n}")
        st.past[b] += n
        row += n
    assert c.past.tolist() == st.past
    return q, out


FORMS = [
    # kv, group, dim, sinks, window, spare slots, calls (new tokens each), causal
    (1, 1, 32, 0, 1, 0, [1, 1, 3], True),
    (2, 2, 64, 4, 10, 0, [1] * 8 + [5, 1, 7], True),
    (2, 4, 64, 4, 33, 3, [40, 1, 1, 17, 2], True),
    (1, 8, 128, 1, 64, 0, [130, 1, 64], True),
    (4, 1, 32, 16, 100, 9, [129, 70, 1], False),
    (2, 3, 64, 5, 70, 0, [20, 65, 1, 90], False),
    (1, 1, 128, 100, 40, 0, [60, 61, 1, 62], True),
    (3, 1, 64, 0, 200, 0, [1, 300, 1], True),
    (1, 16, 64, 2, 300, 0, [290, 1, 2], True),
    (8, 8, 32, 4, 77, 1, [80, 1], False),
]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("kv,group,dim,sinks,window,spare,calls,causal", FORMS)
def test_streams_of_tokens(kind, kv, group, dim, sinks, window, spare, calls, causal):
    note(f"[gpu-test] streams {kind} kv {kv} group {group} dim {dim} sinks {sinks} window {window} {calls} {causal}")
    rng = np.random.default_rng(kv * 1000 + dim + window)
    st = Streams(rng, 2, kv, dim, sinks, sinks + window + max(calls) - 1 + spare, kind)
    for i, n in enumerate(calls):
        run_call(st, n, kv * group, window, causal, even=i % 2 == 1, norm=i % 3 != 2, pad=(0, 8, 1)[i % 3])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_ragged_sequences(kind):
    """Sequences that bring nothing, one token or many, in one call."""
    rng = np.random.default_rng(8)
    st = Streams(rng, 5, 2, 64, 3, 3 + 50 + 80, kind)
    for counts in ([0, 1, 17, 80, 33], [1, 1, 1, 1, 1], [70, 0, 0, 2, 81], [0, 0, 5, 0, 0], [3, 2, 1, 0, 4]):
        run_call(st, 0, 4, 50, True, ragged=counts)


@pytest.mark.parametrize("axes", [(16,), (10, 6), (0, 16, 0), (5, 5, 6)])
def test_axes(axes):
    st = Streams(np.random.default_rng(9), 1, 1, 32, 0, 64, "f32")
    run_call(st, 20, 2, 30, True, sections=axes)
    run_call(st, 3, 2, 30, True, sections=axes, even=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("past", [2 ** 31 - 3, 2 ** 33 + 7])
def test_streams_that_ran_long(kind, past):
    """Positions beyond 32 bits."""
    st = Streams(np.random.default_rng(10), 2, 1, 64, 0, 40, kind, past=[past, past + 1])
    # positions before `past` were never put in: only windows within the new tokens are asked for
    c = st.cache
    run_call(st, 6, 2, 1, True)
    st.base = list(st.base)
    for _ in range(8):
        run_call(st, 5, 2, 2, True)
    assert c.past.tolist() == [past + 46, past + 47]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("batch,heads,kv,dim,window", [(1, 2, 1, 64, 5000), (3, 8, 2, 128, 3001), (2, 4, 4, 32, 9000)])
def test_single_tokens_over_long_windows(kind, batch, heads, kv, dim, window):
    """Few rows over many keys: the keys are split over workgroups."""
    rng = np.random.default_rng(window)
    st = Streams(rng, batch, kv, dim, 4, 4 + window + 9, kind)
    c = st.cache
    # a stream that is past the end of its ring, put in place directly
    past = window + 3000
    for b in range(batch):
        k, v = (normal(rng, (past, kv, dim), KIND[kind]) for _ in range(2))
        st.k[b], st.v[b] = k.double().cpu(), v.double().cpu()
        held = torch.arange(max(0, past - (c.capacity - c.sinks)), past)
        held = torch.cat([torch.arange(c.sinks), held[held >= c.sinks]])
        slots = torch.where(held < c.sinks, held, c.sinks + (held - c.sinks) % (c.capacity - c.sinks)).cuda()
        c.k[b][:, slots] = k[held.cuda()].transpose(0, 1)
        c.v[b][:, slots] = v[held.cuda()].transpose(0, 1)
        st.past[b] = past
    c.seek(st.past)
    for n in (1, 1, 9):
        run_call(st, n, heads, window, True)


def _filled(rng, kind, batch, kv, dim, sinks, capacity, past):
    c = ssc.TokenCache(batch, kv, dim, capacity, sinks=sinks, dtype=kind,
                       k=normal(rng, (batch, kv, capacity, dim), KIND[kind]),
                       v=normal(rng, (batch, kv, capacity, dim), KIND[kind]))
    c.seek([past] * batch)
    return c


def _dense(c, q, window, causal):
    """attend_ref over a cache whose stream never left its first slots."""
    past, n = int(c.past[0]), q.shape[0]
    p = [past + i for i in range(n)]
    last, low = (p if causal else [past + n - 1] * n), [(t if causal else past) - window + 1 for t in p]
    k, v = (t[0, :, :past + n].double().cpu().transpose(0, 1) for t in (c.k, c.v))
    return attend_ref(q.double().cpu(), k, v, p, last, low, c.sinks, c.head_dim ** -0.5, c.dtype, 0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 40, 150])
@pytest.mark.parametrize("causal", [True, False])
def test_infinities_and_nan_behind_the_mask(kind, new, causal):
    """A key that a row does not see leaves no trace in it, whatever it holds;
    rows that see it get what the formula gives."""
    rng = np.random.default_rng(new)
    c = _filled(rng, kind, 1, 2, 64, 2, 400, 200)
    for j, k, v in ((100, math.nan, math.nan), (101, math.inf, math.inf), (102, -math.inf, -math.inf),
                    (199 + new, 1.0, math.inf), (205, 1.0, math.nan), (150, 1.0, -math.inf), (397, math.nan, math.nan)):
        if j < 200 + new or j == 397:
            c.k[0, 1, j, 3], c.v[0, 1, j, 5] = k, v
    q = normal(rng, (new, 4, 64), KIND[kind])
    out = c.attend(q, 60, causal=causal)
    close(out, *_dense(c, q, 60, causal), f"behind the mask {kind} {new} {causal}")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_large_scores(kind):
    """Scores of some hundreds, and rows whose later keys outweigh all before."""
    rng = np.random.default_rng(12)
    c = _filled(rng, kind, 1, 1, 64, 0, 600, 300)
    ramp = torch.linspace(0, 12, 600, device="cuda").to(KIND[kind])
    c.k.mul_(ramp[:, None])
    q = normal(rng, (200, 2, 64), KIND[kind], 4.0)
    close(c.attend(q, 280), *_dense(c, q, 280, True), f"large scores {kind}")


def test_uniform_scores_average():
    """Zero queries: the mean of the values in reach, exactly countable."""
    c = ssc.TokenCache(1, 1, 32, 64, sinks=2, dtype="f32")
    c.v.copy_(torch.arange(64, dtype=torch.float32).view(1, 1, 64, 1).expand(1, 1, 64, 32))
    c.seek([50])
    out = c.attend(torch.zeros(1, 1, 32, device="cuda"), 4)
    assert torch.allclose(out.cpu(), torch.full((1, 1, 32), (0 + 1 + 47 + 48 + 49 + 50) / 6), rtol=1e-6)


def test_a_cache_beyond_32_bits():
    """Slots whose offsets pass 2^31 elements."""
    cap = (1 << 24) + 5000
    k, v = (torch.zeros(1, 1, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = ssc.TokenCache(1, 1, 128, cap, sinks=1, dtype="bf16", k=k, v=v)
    past = cap - 300
    rng = np.random.default_rng(13)
    near = normal(rng, (2, 299, 128), torch.bfloat16)
    k[0, 0, past - 299:past], v[0, 0, past - 299:past] = near[0], near[1]
    c.seek([past])
    qkv = normal(rng, (2, 3 * 128), torch.bfloat16)
    rot = ssc.Rotary(None, (64,))
    pos = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    q = c.append(qkv, pos, rot, 1)
    out = c.attend(q, 200)
    new = qkv.view(2, 3, 128).double().cpu()
    ks = torch.cat([torch.zeros(1, 128, dtype=torch.float64), near[0].double().cpu(), new[:, 1]])[:, None]
    vs = torch.cat([torch.zeros(1, 128, dtype=torch.float64), near[1].double().cpu(), new[:, 2]])[:, None]
    # position 0 (the sink), then past - 299 onwards, as positions 0, 1, ... of a short stream
    ref, tol = attend_ref(q.double().cpu(), ks, vs, None, [300, 301], [101, 102], 1, 128 ** -0.5, "bf16", 0)
    close(out, ref, tol, "far slots")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_results_repeat(kind):
    """Two calls on the same inputs agree bit for bit, also where keys are split."""
    rng = np.random.default_rng(14)
    c = _filled(rng, kind, 3, 2, 64, 4, 5000, 9000)
    for n in (1, 8, 300):
        q = normal(rng, (3 * n, 8, 64), KIND[kind])
        assert torch.equal(c.attend(q, 4600), c.attend(q, 4600))
    x, w = normal(rng, (500, 384), KIND[kind]), normal(rng, (200, 384), KIND[kind])
    assert torch.equal(ssc.linear(x, w), ssc.linear(x, w))
    # a row's result does not depend on the rows beside it
    assert torch.equal(ssc.linear(x, w)[:300], ssc.linear(x[:300], w))


def test_another_stream_than_the_tensors_own():
    rng = np.random.default_rng(15)
    s = torch.cuda.Stream()
    st = Streams(rng, 2, 2, 64, 2, 60, "bf16")
    for n in (20, 1, 5):
        run_call(st, n, 4, 30, True, stream=s)
    x, w = normal(rng, (300, 128), torch.bfloat16), normal(rng, (64, 128), torch.bfloat16)
    y = ssc.linear(x * 2, w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    close(y, *linear_ref(x * 2, w, None, "none", None, "bf16"), "other stream")


def test_refused_on_the_device_side():
    rng = np.random.default_rng(16)
    c = _filled(rng, "bf16", 1, 1, 64, 2, 100, 500)
    q = normal(rng, (1, 2, 64), torch.bfloat16)
    with pytest.raises(ssc.SscaterError) as e:
        c.attend(q, 99)                       # 98 ring slots
    assert e.value.code == ssc.E_INVALID_ARG
    c.attend(q, 98)
    with pytest.raises(ValueError):
        c.attend(q.float(), 10)
    with pytest.raises(ValueError):
        c.attend(q[:, :, :32], 10)
    with pytest.raises(ValueError):
        c.append(q.view(1, 128), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), ssc.Rotary(None, (32,)), 2)
    with pytest.raises(ValueError):
        ssc.linear(q[0], normal(rng, (8, 65), torch.bfloat16))
    with pytest.raises(ValueError):
        ssc.linear(q[0], normal(rng, (8, 64), torch.float32))
    with pytest.raises(ValueError):
        ssc.linear(q[0].t().contiguous().t(), normal(rng, (8, 64), torch.bfloat16))


def test_a_captured_step_replays():
    """Append, attend, linear and advance in a graph: replays advance the stream
    as eager calls do, with other work between them."""
    rng = np.random.default_rng(17)
    kind, heads, kv, dim, window, n = torch.bfloat16, 4, 2, 64, 3000, 2
    make = lambda: ssc.TokenCache(1, kv, dim, 4 + window + n - 1, sinks=4, dtype="bf16")  # noqa: E731
    rot = ssc.Rotary(None, (16, 8, 8))
    w = normal(rng, (heads * dim, heads * dim), kind, 0.05)
    qkv = torch.empty(n, (heads + 2 * kv) * dim, dtype=kind, device="cuda")
    pos = torch.empty(n, 3, dtype=torch.int32, device="cuda")

    def step(c):
        o = c.attend(c.append(qkv, pos, rot, heads), window)
        y = ssc.linear(o.view(n, -1), w, activation="silu")
        c.advance(n)
        return y

    data = [(normal(rng, qkv.shape, kind), torch.from_numpy(rng.integers(0, 900, (n, 3)).astype(np.int32)).cuda())
            for _ in range(6)]
    eager, graphed = make(), make()
    for c in (eager, graphed):
        c.k.copy_(normal(np.random.default_rng(18), c.k.shape, kind))
        c.v.copy_(normal(np.random.default_rng(19), c.v.shape, kind))
        c.seek([5000])
    want = []
    for a, p in data:
        qkv.copy_(a)
        pos.copy_(p)
        want.append(step(eager).clone())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        y = step(graphed)
    torch.cuda.synchronize()
    graphed.k.copy_(normal(np.random.default_rng(18), graphed.k.shape, kind))
    graphed.v.copy_(normal(np.random.default_rng(19), graphed.v.shape, kind))
    graphed.seek([5000])
    for i, (a, p) in enumerate(data):
        qkv.copy_(a)
        pos.copy_(p)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i]), f"replay {i}"
        torch.randn(1000, device="cuda").sum().item()
    assert graphed.past.tolist() == eager.past.tolist() == [5012]
    assert torch.equal(graphed.k, eager.k) and torch.equal(graphed.v, eager.v)
