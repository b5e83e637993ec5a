"""GPU tests of the gated delta rule with infinite queries that are taken as they are."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_delta import Case, bound  # noqa: E402


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,at", [(3, 1), (150, 0), (150, 70), (150, 149), (1500, 700), (1500, 1499)])
@pytest.mark.parametrize("value", [math.inf, -math.inf])
def test_an_infinite_query_reads_the_sign_of_the_state(value, n, at, kind):
    """out = scale S^T q: the infinity's sign times that of the state's row; no other token's."""
    c = Case(21, [n], 2, 1, 64, 32, kind, raw=False, unit=False)
    (_, _, S, err, ref, tol), = c.sequences()
    # the state after token `at`: what unit queries read there, in 64 bits
    part = Case(21, [n], 2, 1, 64, 32, kind, raw=False, unit=False)
    for name in "qkvab":
        setattr(part, name, getattr(part, name)[:at + 1])
    part.counts = [at + 1]
    (_, _, then, wide, _, _), = part.sequences()
    c.q[at, 0, 5] = value
    out = c.call()
    sure = then[:, 5].abs() > wide + 1e-6
    assert float(sure.double().mean()) > 0.9
    want = torch.sign(then[:, 5]) * value
    assert torch.equal(out[at].double().cpu()[sure], want[sure])
    rest = [i for i in range(n) if i != at]
    bound(out[rest], ref[rest], tol[rest], "the other tokens")
    assert bool(((c.memory.state[0].double().cpu() - S).norm(dim=1) <= err + 2 * 2.0 ** -24 * S.norm(dim=1)).all())
