"""GPU tests of the query decoder over maps without a cell."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2512_08557_amd import QueryDecoder  # noqa: E402
from test_gpu_decoder import C, CELLS, DIM, DK, DV, KV, MH, QH, QK, QUERIES, make_weights  # noqa: E402


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch", [1, 3])
def test_a_stride_without_cells_is_one_whose_cells_are_hidden(batch, kind):
    w = make_weights(np.random.default_rng(5), kind)
    one, two = (QueryDecoder(w, QUERIES, MH, DK, DV, QH, KV, DIM, qk_heads=QK, batch=batch) for _ in range(2))
    a = b = torch.randn(batch, QUERIES, C, device="cuda").to(kind)
    cells = torch.randn(batch, 70, CELLS, device="cuda").to(kind)
    hidden = torch.zeros(batch, 70, dtype=torch.bool, device="cuda")
    for stride in range(3):
        if stride == 1:
            a, ya = one.step(a, cells)
            b, yb = two.step(b, cells)
        else:
            a, ya = one.step(a, cells[:, :0], hidden[:, :0].contiguous() if stride else None)
            b, yb = two.step(b, cells, hidden)
        assert torch.equal(a, b) and torch.equal(ya, yb), f"stride {stride}"
        assert torch.equal(one.memory.state, two.memory.state)
