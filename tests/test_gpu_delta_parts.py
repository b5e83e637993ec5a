"""GPU tests of the gated delta rule over streams that are taken in parts, where a part's
own transition is large, infinite or NaN and the memory is not: what comes out is the
recurrence's, as for short streams and token by token.  Tolerances as in
test_gpu_delta.py: they hold as long as the tokens from the first that is remembered on
do not lengthen a column."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_delta import Case  # noqa: E402


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (32, 128), (128, 32), (128, 128)])
@pytest.mark.parametrize("n", [200, 700, 1500, 3348])
def test_an_empty_memory_stays_empty(n, dk, dv, kind):
    """Values of zeros with keys whose transitions grow from token to token."""
    c = Case(31, [n, 90], 2, 1, dk, dv, kind, raw=False, unit=False)
    c.k.mul_(2 * dk ** 0.5)
    c.v.zero_()
    c.memory.state.zero_()
    out = c.call(start=c.start, max_new=n)
    assert not bool(out.ne(0).any()) and not bool(c.memory.state.ne(0).any())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (32, 128), (128, 32)])
@pytest.mark.parametrize("n,at", [(150, 70), (500, 200), (1500, 0), (1500, 700), (3348, 1000), (3348, 3300)])
def test_a_large_key_on_an_empty_memory(n, at, dk, dv, kind):
    """Finite with the tokens one after the other, though the key's square is not."""
    c = Case(32, [n], 2, 1, dk, dv, kind, raw=False, unit=False)
    c.v.zero_()
    c.v[at] = 1.0
    c.k[at] = 1e22
    c.state.zero_()
    c.memory.state.zero_()
    c.check()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", [[3000, 70, 0, 1500], [2000, 1999]])
def test_other_streams_and_heads_are_as_they_were(lengths, kind):
    """A transition that overflows in one head of one stream."""
    want = Case(33, lengths, 4, 4, 64, 64, kind, raw=False, unit=False)
    ref = want.call(start=want.start, max_new=lengths[0]).clone()
    c = Case(33, lengths, 4, 4, 64, 64, kind, raw=False, unit=False)
    c.state[0, 2].zero_()
    c.memory.state[0, 2].zero_()
    c.v[:lengths[0], 2].zero_()
    c.k[:lengths[0], 2] *= 60
    out = c.call(start=c.start, max_new=lengths[0])
    assert not bool(out[:lengths[0], 2].ne(0).any()) and not bool(c.memory.state[0, 2].ne(0).any())
    same = torch.ones_like(out, dtype=torch.bool)
    same[:lengths[0], 2] = False
    assert torch.equal(out[same], ref[same])
    same = torch.ones_like(c.memory.state, dtype=torch.bool)
    same[0, 2] = False
    assert torch.equal(c.memory.state[same], want.memory.state[same])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("at", [100, 700, 1400])
def test_a_key_that_is_no_number(at, kind):
    """A NaN in a key is every later output's, and none of the ones before it."""
    c = Case(34, [1500], 2, 1, 64, 32, kind)
    (_, s, _, _, ref, tol), = c.sequences()
    c.k[at, 0, 5] = math.nan
    out = c.call()
    good = out[:at].double().cpu()
    assert bool(((good - ref[:at]).abs() <= tol[:at]).all())
    assert not bool(torch.isfinite(out[at:]).any()) and not bool(torch.isfinite(c.memory.state).any())

