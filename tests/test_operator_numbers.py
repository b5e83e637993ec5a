"""Scales and eps of the token and decoder operators on the host: a call takes what they
hold when it is made.  Tensors of the CPU that pass for cuda ones, and a library call
that only looks at its description: nothing reaches a GPU."""
import pytest

torch = pytest.importorskip("torch")

import paper_2512_08557_amd as ssc  # noqa: E402
from paper_2512_08557_amd import tokens as T  # noqa: E402


class Fake(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def fake(*shape):
    return torch.zeros(shape).as_subclass(Fake)


@pytest.fixture
def seen(monkeypatch):
    """The descriptions of the calls."""
    specs = []
    monkeypatch.setattr(T, "_launch", lambda fn, where, index, stream, tensors, spec, *args: specs.append(spec))
    T._bind()
    return specs


def norm(eps):
    ssc.norm(fake(4, 32), eps=eps)


def add_norm(eps):
    ssc.add_norm(fake(4, 32), fake(4, 32), fake(32), eps=eps)


def cross(scale):
    q = fake(2, 40, 4, 32)
    ssc.cross_attend(q, q, q, scale=scale)


def ragged(scale):
    q, start = fake(40, 4, 32), torch.tensor([0, 3, 40], dtype=torch.int32).as_subclass(Fake)
    ssc.cross_attend(q, q, q, q_start=start, k_start=start, scale=scale)


def delta(**number):
    m = ssc.DeltaMemory(2, 4, 32, 32, state=fake(2, 4, 32, 32))
    q, a = fake(6, 4, 32), fake(6, 4)
    m.update(q, q, q, a, a, **number)


def attend(scale):
    k = fake(2, 4, 64, 32)
    c = ssc.TokenCache(2, 4, 32, 64, k=k, v=k)
    c.attend(fake(2, 4, 32), 5, scale=scale)


CALLS = [(norm, "eps"), (add_norm, "eps"), (cross, "scale"), (ragged, "scale"), (lambda eps: delta(eps=eps), "eps"),
         (lambda scale: delta(scale=scale), "scale"), (attend, "scale")]


@pytest.mark.parametrize("call,field", CALLS)
def test_a_number_that_changes_between_two_calls(call, field, seen):
    for make in (torch.tensor, lambda v: torch.tensor([v])[0]):
        number = make(0.5)
        call(number)
        number.fill_(2.0)
        call(number)
        assert [getattr(s, field) for s in seen[-2:]] == [0.5, 2.0]
    for value in (0.25, 1, True):
        call(value)
        assert getattr(seen[-1], field) == value


@pytest.mark.parametrize("call,field", CALLS)
def test_a_number_that_wants_a_gradient(call, field, seen):
    number = torch.nn.Parameter(torch.tensor(0.5))
    with pytest.raises(ValueError, match="gradient"):
        call(number)
    assert not seen
    with torch.no_grad():
        call(number)
        number.fill_(2.0)
        call(number)
    assert [getattr(s, field) for s in seen] == [0.5, 2.0]
