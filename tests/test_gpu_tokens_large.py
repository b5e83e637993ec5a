"""GPU tests of token operator calls that are more threads than one launch takes
(2^32), on some tens of gigabytes."""
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2512_08557_amd as ssc  # noqa: E402


def test_append_of_many_tokens():
    """2^26 + 5 tokens of one stream; the cache keeps the last ones."""
    tokens, dim, capacity = (1 << 26) + 5, 32, 40
    note(f"[gpu-test] append {tokens}")
    gen = torch.Generator("cuda").manual_seed(1)
    qkv = torch.empty(tokens, 3 * dim, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    pos = torch.zeros(tokens, 1, dtype=torch.int32, device="cuda")
    c = ssc.TokenCache(1, 1, dim, capacity, sinks=4, dtype="bf16")
    # position 0: every head as it was
    q = c.append(qkv, pos, ssc.Rotary(None, (dim // 2,)), 1)
    for part in range(0, tokens, 1 << 24):
        assert torch.equal(q[part:part + (1 << 24), 0], qkv[part:part + (1 << 24), :dim]), part
    held = torch.cat([torch.arange(4), torch.arange(tokens - 36, tokens)])
    slot = torch.where(held < 4, held, 4 + (held - 4) % 36).cuda()
    held = held.cuda()
    assert torch.equal(c.k[0, 0, slot], qkv[held, dim:2 * dim]) and torch.equal(c.v[0, 0, slot], qkv[held, 2 * dim:])
    c.advance(tokens)
    assert c.past.tolist() == [tokens]


def test_attention_of_many_streams():
    """2^23 streams with one key each, two heads: the values themselves."""
    batch = 1 << 23
    note(f"[gpu-test] attend {batch}")
    gen = torch.Generator("cuda").manual_seed(2)
    make = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)  # noqa: E731
    c = ssc.TokenCache(batch, 2, 32, 1, dtype="bf16", k=make(batch, 2, 1, 32), v=make(batch, 2, 1, 32))
    assert torch.equal(c.attend(make(batch, 2, 32), 1), c.v[:, :, 0])


def test_linear_over_many_rows():
    """2^31 + 300 rows of one channel: one product each, rounded once."""
    rows, part = (1 << 31) + 300, 1 << 28
    note(f"[gpu-test] linear {rows}")
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w = torch.full((1, 1), 1.3, dtype=torch.bfloat16, device="cuda")
    y = ssc.linear(x, w)
    for i in range(0, rows, part):
        assert torch.equal(y[i:i + part], (x[i:i + part].float() * w.float()).to(torch.bfloat16)), i


def test_linear_over_many_channels():
    """2^24 channels of a few rows, in parts of the layer: products, biases and
    residuals (whole numbers, so every sum is exact) meet their own."""
    channels = (1 << 24) + 72
    note(f"[gpu-test] linear to {channels}")
    i = torch.arange(channels, device="cuda")
    x = torch.arange(1, 71, device="cuda").float()[:, None]
    w, b = (i * 37 % 251 - 125).float()[:, None], (i * 11 % 1009).float()
    r = (torch.arange(70 * channels, device="cuda").view(70, channels) * 7 % 2003).float()
    assert torch.equal(ssc.linear(x, w, b, residual=r), x * w.t() + b + r)
