"""Operands, memories and outputs that want a gradient are refused on the host by every
token and decoder operator, and taken under no_grad.  (Tensors of the CPU that pass for
cuda ones: nothing reaches a GPU.)"""
import pytest

torch = pytest.importorskip("torch")

import paper_2512_08557_amd as ssc  # noqa: E402
from test_operator_numbers import Fake, fake, seen  # noqa: E402,F401


def norm(t):
    ssc.norm(t("x", 4, 32), t("weight", 32), t("bias", 32), gate=t("gate", 4, 32), out=t("out", 4, 32))


def add_norm(t):
    ssc.add_norm(t("x", 4, 32), t("block", 4, 32), t("weight", 32), t("bias", 32), block_weight=t("block_weight", 32),
                 block_bias=t("block_bias", 32), gate=t("gate", 4, 32), scale=t("scale", 32), total=t("total", 4, 32),
                 out=t("out", 4, 32))


def cross(t):
    ssc.cross_attend(t("q", 2, 5, 4, 32), t("k", 2, 9, 4, 32), t("v", 2, 9, 4, 32), out=t("out", 2, 5, 4, 32))


def delta(t):
    m = ssc.DeltaMemory(2, 4, 32, 32, state=t("state", 2, 4, 32, 32))
    m.update(t("q", 6, 4, 32), t("k", 6, 4, 32), t("v", 6, 4, 32), t("a", 6, 4), t("b", 6, 4), rate=t("rate", 4), bias=t("bias", 4),
             initial=t("initial", 2, 4, 32, 32), out=t("out", 6, 4, 32))


def linear(t):
    ssc.linear(t("x", 4, 32), t("weight", 8, 32), t("bias", 8), residual=t("residual", 4, 8), out=t("out", 4, 8))


def append(t):
    c = ssc.TokenCache(2, 2, 32, 64, k=t("k", 2, 2, 64, 32), v=t("v", 2, 2, 64, 32))
    rotary = ssc.Rotary(fake(16), [16])
    c.append(t("qkv", 6, 8 * 32), torch.zeros(6, 1, dtype=torch.int32).as_subclass(Fake), rotary, 4, q_weight=t("q_weight", 32),
             k_weight=t("k_weight", 32), out=t("out", 6, 4, 32))


def attend(t):
    c = ssc.TokenCache(2, 2, 32, 64, k=t("k", 2, 2, 64, 32), v=t("v", 2, 2, 64, 32))
    c.attend(t("q", 6, 4, 32), 5, out=t("out", 6, 4, 32))


CALLS = [(norm, "x weight bias gate out"), (add_norm, "x block weight bias block_weight block_bias gate scale total out"),
         (cross, "q k v out"), (delta, "state q k v a b rate bias initial out"), (linear, "x weight bias residual out"),
         (append, "k v qkv q_weight k_weight out"), (attend, "k v q out")]


@pytest.mark.parametrize("call,which", [(c, n) for c, names in CALLS for n in names.split()])
def test_what_wants_a_gradient_is_refused(call, which, seen):  # noqa: F811
    def t(name, *shape):
        return fake(*shape).requires_grad_(name == which)
    with pytest.raises(ValueError, match="gradient"):
        call(t)
    assert not seen
    with torch.no_grad():
        call(t)
    assert len(seen) == 1
