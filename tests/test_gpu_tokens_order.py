"""GPU tests of what the attention's results may not depend on."""
import math

import numpy as np
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2512_08557_amd as ssc  # noqa: E402

KIND = {"f32": torch.float32, "bf16": torch.bfloat16}


def normal(rng, shape, kind, std=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(kind).cuda()


def filled(rng, kind, kv, dim, capacity, past, batch=1):
    c = ssc.TokenCache(batch, kv, dim, capacity, dtype=kind, k=normal(rng, (batch, kv, capacity, dim), KIND[kind]),
                       v=normal(rng, (batch, kv, capacity, dim), KIND[kind]))
    c.seek([past] * batch)
    return c


def leave(value):
    """A layer over so many rows that its tiles go through the LDS of every
    compute unit, which then holds `value` and sums of it."""
    x = torch.full((256 * 256, 192), value, dtype=torch.bfloat16, device="cuda")
    ssc.linear(x, torch.full((128, 192), value, dtype=torch.bfloat16, device="cuda"))


# Rows of one key head (q_heads = rows, one token) and keys.  33 to 64 rows, and
# fp32 heads of 128 from one row on, share a workgroup with a second group of
# keys, which has no tile in the last round where the tiles of 64 (bf16) or 32
# (fp32) keys are odd in number.
@pytest.mark.parametrize("kind,dim,rows,keys", [
    ("bf16", 32, 40, 150), ("bf16", 64, 33, 60), ("bf16", 64, 48, 128), ("bf16", 64, 64, 192), ("bf16", 128, 50, 180),
    ("bf16", 64, 40, 700), ("f32", 32, 40, 90), ("f32", 64, 64, 96), ("f32", 64, 33, 30), ("f32", 128, 1, 32),
    ("f32", 128, 1, 64), ("f32", 128, 1, 96), ("f32", 128, 40, 160), ("bf16", 64, 8, 130), ("bf16", 64, 100, 130),
    ("f32", 64, 100, 130)])
def test_results_do_not_depend_on_what_ran_before(kind, dim, rows, keys):
    note(f"[gpu-test] after other kernels {kind} dim {dim} rows {rows} keys {keys}")
    rng = np.random.default_rng(rows * 1000 + keys + dim)
    c = filled(rng, kind, 1, dim, keys, keys - 1)
    q = normal(rng, (1, rows, dim), KIND[kind], 2.0)
    leave(1.0)
    want = c.attend(q, keys)
    for value in (math.inf, math.nan, -math.inf, 2.0 ** 100):
        leave(value)
        assert torch.equal(c.attend(q, keys), want), f"after a kernel over {value}"


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,dim,new,heads", [("bf16", 64, 1, 8), ("bf16", 64, 12, 4), ("bf16", 128, 50, 4),
                                                ("bf16", 32, 200, 1), ("f32", 64, 12, 2), ("f32", 64, 40, 1),
                                                ("f32", 32, 200, 2), ("f32", 128, 8, 4)])
def test_a_row_does_not_depend_on_the_other_rows(kind, dim, new, heads, causal):
    """A query forty times as large moves its own row's exponents and no other
    row's bits."""
    note(f"[gpu-test] other rows {kind} dim {dim} new {new} heads {heads} causal {causal}")
    rng = np.random.default_rng(new * 10 + heads)
    c = filled(rng, kind, 1, dim, 900, 700)
    q = normal(rng, (new, heads, dim), KIND[kind], 2.0)
    want = c.attend(q, 600, causal=causal)
    for t, h in {(0, 0), (new // 2, heads - 1), (new - 1, 0)}:
        other = q.clone()
        other[t, h] *= 40
        got = c.attend(other, 600, causal=causal)
        got[t, h] = want[t, h]
        assert torch.equal(got, want), f"query {t}, {h}"
