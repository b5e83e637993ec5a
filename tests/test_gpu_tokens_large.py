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
