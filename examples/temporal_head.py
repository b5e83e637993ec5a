"""Backbone, temporal block and head on a synthetic sweep: one line per stride.

    python examples/temporal_head.py [strides]

The 432x496 backbone (fp32) is advanced stride by stride; its last map's 62 x 54
cells of 256 channels attend to those of the last ten strides and go through a
feed-forward layer, and a 1x1 head gives 42 values per cell.  All weights are
random: the example shows the calls and what they cost.
"""
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import streams as S  # noqa: E402
from paper_2512_08557_amd import Engine, TemporalBlock, linear  # noqa: E402


def main(strides: int = 12) -> None:
    wl = S.workload("c3")
    layers = [(l.cin, l.cout, l.stride, l.relu) for l in wl.layers]
    eng = Engine(wl.H, wl.W, wl.C0, layers, S.weights("c3"), dtype=wl.dtype, max_pillars=wl.max_pillars)
    last = len(layers)
    h, w, c = eng.shapes[last]
    heads, dim, inner, outputs = 8, 32, 4 * c, 42
    gen = torch.Generator("cuda").manual_seed(7)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda") * s[-1] ** -0.5  # noqa: E731
    one = torch.ones(dim, device="cuda")
    block = TemporalBlock({"qkv": rand(3 * heads * dim, c), "q_norm": one, "k_norm": one, "out": rand(c, heads * dim),
                           "up": rand(inner, c), "up_bias": torch.zeros(inner, device="cuda"), "down": rand(c, inner)},
                          heads, heads, dim, tokens=h * w, strides=10)
    w_head, b_head = rand(outputs, c), torch.zeros(outputs, device="cuda")
    for st in S.make_stream("c3", n_strides=strides):
        idx, feats = torch.from_numpy(st.idx).cuda(), torch.from_numpy(st.feats).cuda()
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        eng.step(idx, feats, sorted=True)
        x = eng.read(last).view(-1, c)
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        y = linear(block.step(x, st.index, (h, w)), w_head, b_head)
        torch.cuda.synchronize()
        t2 = time.perf_counter()
        print(f"stride {st.index}: backbone {1e6 * (t1 - t0):.0f} us, temporal block and head {1e6 * (t2 - t1):.0f} us, "
              f"output {tuple(y.shape)}, finite {bool(torch.isfinite(y).all())}", flush=True)
    eng.close()


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 12)
