"""GPU tests of masks over more keys than a list's workgroups count for themselves.

Outputs against those of the visible keys gathered by the caller, in 64 bits: scores are
off by 2 (sqrt(D) + 8) u scale sum |q k| and 4 u of themselves before exp (u = 2^-24),
twice, sums of n terms by 2 (sqrt(n) + 8) u, all relative to sum p |v|, and the output by
2 u of itself."""
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


def normal(rng, shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()


def check(got, q, k, v, seen, what):
    """One sequence, one key head."""
    got, q = got.double().cpu(), q.double().cpu()
    k, v = k[seen].double().cpu()[:, 0], v[seen].double().cpu()[:, 0]
    if len(k) == 0:
        assert float(got.abs().sum()) == 0.0, what
        return
    for h in range(q.shape[1]):
        x = q[:, h]
        s = x @ k.t() / math.sqrt(32)
        p = torch.softmax(s, -1)
        ref = p @ v
        err = 2 * (math.sqrt(32) + 8) * U * (x.abs() @ k.abs().t()) / math.sqrt(32) + 4 * U * s.abs()
        tol = (2 * err.max(-1, keepdim=True).values + 2 * (math.sqrt(len(k)) + 8) * U) * (p @ v.abs()) + 2 * U * ref.abs()
        worst = float(((got[:, h] - ref).abs() / tol).max())
        note(f"[gpu-test] {what} head {h}: {worst:.3f} of the tolerance")
        assert worst <= 1.0, f"{what}: {worst}"


@pytest.mark.parametrize("queries", [1, 40, 200])
@pytest.mark.parametrize("keys", [262144, 262145, 300001, 999999])
def test_one_long_sequence(keys, queries):
    """Either side of the largest list without counts; masks of runs, single keys and none."""
    note(f"[gpu-test] {queries} queries to {keys} masked keys")
    rng = np.random.default_rng(keys + queries)
    q, k, v = normal(rng, (queries, 2, 32)), normal(rng, (keys, 1, 32)), normal(rng, (keys, 1, 32))
    masks = [rng.random(keys) < 0.01, np.arange(keys) == keys - 1, np.arange(keys) % 4096 == 4095, np.zeros(keys, bool),
             (np.arange(keys) < 70000) & (rng.random(keys) < 0.5), np.arange(keys) >= keys - 5000]
    for i, m in enumerate(masks):
        seen = torch.from_numpy(m).cuda()
        check(ssc.cross_attend(q, k, v, seen), q, k, v, seen, f"mask {i}")


@pytest.mark.parametrize("queries", [2, 50])
def test_sequences_of_different_lengths(queries):
    """Long ones among short and empty ones, beginning anywhere; rows behind the last."""
    rng = np.random.default_rng(queries)
    nk, nq = [5, 0, 300007, 4096, 1, 270000, 0, 33], [queries, 1, queries, 0, 1, queries, 2, 1]
    q, k, v = normal(rng, (sum(nq) + 3, 2, 32)), normal(rng, (sum(nk) + 9, 1, 32)), normal(rng, (sum(nk) + 9, 1, 32))
    seen = torch.from_numpy(rng.random(sum(nk) + 9) < 0.02).cuda()
    seen[5:9] = True
    seen[sum(nk):] = True
    k[sum(nk):] = math.nan
    starts = [torch.tensor([0] + list(np.cumsum(n)), dtype=torch.int32).cuda() for n in (nq, nk)]
    for limits in (dict(max_q=max(nq), max_k=max(nk)), {}):
        out = torch.full_like(q, 7.0)
        ssc.cross_attend(q, k, v, seen, *starts, out=out, **limits)
        assert bool((out[sum(nq):] == 7.0).all())
        a = c = 0
        for b, (n, m) in enumerate(zip(nq, nk)):
            if n:
                check(out[a:a + n], q[a:a + n], k[c:c + m], v[c:c + m], seen[c:c + m], f"sequence {b}")
            a, c = a + n, c + m


@pytest.mark.parametrize("batch,most", [(20000, 40), (3000, 120), (100000, 3), (150, 1400), (40, 9000)])
def test_many_sequences_whose_longest_is_not_known(batch, most):
    """The most of one sequence is taken to be all; counted first and not."""
    note(f"[gpu-test] {batch} masked sequences of less than {most} keys")
    rng = np.random.default_rng(5)
    nk = rng.integers(0, most, batch)
    total = int(nk.sum())
    q, k, v = normal(rng, (batch, 1, 32)), normal(rng, (total, 1, 32)), normal(rng, (total, 1, 32))
    seen = torch.from_numpy(rng.random(total) < 0.3).cuda()
    starts = [torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).cuda() for n in (np.ones(batch, np.int64), nk)]
    out = ssc.cross_attend(q, k, v, seen, *starts, max_q=1)
    want = ssc.cross_attend(q, k, v, seen, *starts, max_q=1, max_k=most - 1)
    at = np.concatenate([[0], np.cumsum(nk)])
    for b in list(range(0, batch, batch // 8)) + [batch - 1]:
        s = slice(int(at[b]), int(at[b + 1]))
        check(out[b:b + 1], q[b:b + 1], k[s], v[s], seen[s], f"sequence {b}")
    none = torch.tensor([not bool(x) for x in np.add.reduceat(np.append(seen.cpu().numpy(), False), at[:-1]) * (nk > 0)])
    assert float(out[none.cuda()].abs().sum()) == 0.0
    assert float((out - want).abs().max()) <= 1e-5


def test_a_long_mask_is_read_a_few_times():
    """2^28 keys, one in 65536 visible: three passes over 268 MB of mask.  Counted once
    for each of its 65536 parts it would be 8.8e12 bytes, half a second at 16 TB/s."""
    n = 1 << 28
    rng = np.random.default_rng(6)
    k = torch.zeros((n, 1, 32), dtype=torch.bfloat16, device="cuda")
    seen = torch.zeros(n, dtype=torch.bool, device="cuda")
    at = torch.arange(0, n, 65536, device="cuda") + torch.from_numpy(rng.integers(0, 65536, n // 65536)).cuda()
    k[at] = normal(rng, (len(at), 1, 32)).bfloat16()
    seen[at] = True
    q = normal(rng, (1, 1, 32)).bfloat16()
    out = ssc.cross_attend(q, k, k, seen)
    want = ssc.cross_attend(q, k[at], k[at])
    assert bool(torch.isfinite(out).all()) and float((out - want).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    ssc.cross_attend(q, k, k, seen)
    end.record()
    torch.cuda.synchronize()
    note(f"[gpu-test] 2^28 masked keys: {begin.elapsed_time(end):.2f} ms")
    assert begin.elapsed_time(end) < 100


def test_a_captured_call_replays():
    rng = np.random.default_rng(7)
    q, k, v = normal(rng, (5, 1, 32)), normal(rng, (280000, 1, 32)), normal(rng, (280000, 1, 32))
    masks = [torch.from_numpy(rng.random(280000) < p).cuda() for p in (0.5, 0.0, 0.01, 1.0)]
    want = [ssc.cross_attend(q, k, v, m) for m in masks]
    seen = masks[0].clone()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        out = ssc.cross_attend(q, k, v, seen)
    for i in (0, 1, 2, 3, 1, 0):
        seen.copy_(masks[i])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i]), f"replay {i}"
        torch.randn(1000, device="cuda").sum().item()
