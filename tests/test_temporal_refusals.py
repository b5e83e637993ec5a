"""What TemporalBlock refuses when it is made, on any machine."""
import pytest

torch = pytest.importorskip("torch")

from paper_2512_08557_amd import TemporalBlock  # noqa: E402


def weights(dtype):
    make = lambda *s: torch.zeros(*s, dtype=dtype)  # noqa: E731
    return {"qkv": make(96, 32), "q_norm": make(32), "k_norm": make(32), "out": make(32, 32), "up": make(64, 32),
            "down": make(32, 64)}


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int32])
def test_other_types_are_refused(dtype):
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        TemporalBlock(weights(dtype), 1, 1, 32, tokens=4, strides=2)


@pytest.mark.parametrize("name", ["q_norm", "down", "up_bias"])
def test_mixed_types_are_refused(name):
    w = dict(weights(torch.float32), up_bias=torch.zeros(64))
    w[name] = w[name].bfloat16()
    with pytest.raises(ValueError, match=name):
        TemporalBlock(w, 1, 1, 32, tokens=4, strides=2)


def test_absent_biases_and_further_entries_are_no_matter():
    w = dict(weights(torch.float32), up_bias=None, out_bias=torch.zeros(32), head=torch.zeros(4, 32).half())
    # everything but the device is right
    with pytest.raises(ValueError, match="cuda tensor"):
        TemporalBlock(w, 1, 1, 32, tokens=4, strides=2)
