"""GPU tests of which calls the token operators refuse, and of what a refused one leaves."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2512_08557_amd as ssc  # noqa: E402


def test_operands_that_want_a_gradient_are_refused():
    """No gradient is formed: a result that silently has none would be taken for
    a constant."""
    x, w = torch.randn(4, 32, device="cuda"), torch.randn(8, 32, device="cuda")
    b, r = torch.randn(8, device="cuda"), torch.randn(4, 8, device="cuda")
    want = ssc.linear(x, w, b, residual=r)
    for at in range(4):
        ops = [t.clone().requires_grad_(i == at) for i, t in enumerate((x, w, b, r))]
        with pytest.raises(ValueError, match="gradient"):
            ssc.linear(ops[0], ops[1], ops[2], residual=ops[3])
        with torch.no_grad():
            assert torch.equal(ssc.linear(ops[0], ops[1], ops[2], residual=ops[3]), want)
    c = ssc.TokenCache(1, 1, 32, 8)
    qkv, pos = torch.randn(2, 96, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    one = torch.ones(32, device="cuda")
    rot = ssc.Rotary(None, (16,))
    with pytest.raises(ValueError, match="gradient"):
        c.append(qkv.clone().requires_grad_(), pos, rot, 1)
    for qw, kw in ((one.clone().requires_grad_(), one), (one, one.clone().requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            c.append(qkv, pos, rot, 1, q_weight=qw, k_weight=kw)
    q = c.append(qkv, pos, rot, 1, q_weight=one, k_weight=one)
    with pytest.raises(ValueError, match="gradient"):
        c.attend(q.clone().requires_grad_(), 4)
    with torch.no_grad():
        assert torch.equal(c.attend(q.clone().requires_grad_(), 4), c.attend(q, 4))


def test_a_stride_of_too_many_cells_leaves_the_block_as_it_was():
    rng = np.random.default_rng(3)
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32) * s[-1] ** -0.5).cuda()  # noqa: E731
    w = {"qkv": make(3 * 64, 32), "q_norm": torch.ones(32).cuda(), "k_norm": torch.ones(32).cuda(),
         "out": make(32, 64), "up": make(96, 32), "down": make(32, 96)}
    one, two = (ssc.TemporalBlock(w, 2, 2, 32, tokens=9, strides=2, sinks=1) for _ in range(2))
    for stride in range(8):
        x = make(9, 32)
        if stride in (0, 5):
            with pytest.raises(ValueError, match="9"):
                two.step(make(16, 32), stride, (4, 4))
        assert torch.equal(one.step(x, stride, (3, 3)), two.step(x, stride, (3, 3))), f"stride {stride}"
