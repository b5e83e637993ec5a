"""GPU tests of layers of few channels over many rows, whose tiles hold all
channels, on either side of where they begin; tolerances as for all layers."""
import numpy as np
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2512_08557_amd as ssc  # noqa: E402
from test_gpu_tokens import KIND, close, linear_ref, normal  # noqa: E402


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cin,cout,pad", [(32767, 16, 42, 0), (32768, 16, 42, 0), (33001, 40, 42, 0),
                                               (32769, 33, 7, 0), (40000, 72, 64, 0), (32800, 24, 64, 1),
                                               (32900, 9, 1, 0), (33333, 200, 33, 3), (50000, 8, 50, 6)])
def test_few_channels_over_many_rows(rows, cin, cout, pad, kind):
    note(f"[gpu-test] linear {rows} {cin} {cout} pad {pad} {kind}")
    rng = np.random.default_rng(rows + cin + cout)
    x, w = normal(rng, (rows, cin), KIND[kind]), normal(rng, (cout, cin), KIND[kind], cin ** -0.5)
    b, r = normal(rng, (cout,), KIND[kind]), normal(rng, (rows, cout), KIND[kind])
    flat = normal(rng, (rows, cout + pad), KIND[kind])
    before, out = flat.clone(), flat[:, :cout]
    for act, bias, res in (("gelu", b, None), ("relu", None, r), ("none", b, r)):
        y = ssc.linear(x, w, bias, activation=act, residual=res, out=out)
        close(y, *linear_ref(x, w, bias, act, res, kind), act)
        assert torch.equal(flat[:, cout:], before[:, cout:])
