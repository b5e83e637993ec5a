"""Host-side argument checks of the norms, cross attention and the delta memory: every
bad call is refused before any HIP work, so the pointers here are never dereferenced."""
import ctypes

import pytest

import paper_2512_08557_amd as ssc
from paper_2512_08557_amd import engine as E

P = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 1)
OFF = ctypes.c_void_p((1 << 20) + 4)


def _norm(at=None, ptr=None, ptrs=None, **kw):
    f = dict(rows=4, gate_rows=2, width=8, dtype=E.F32, center=0, block_norm=1, activation=3, eps=1e-6, x_stride=8,
             block_stride=8, gate_stride=8, sum_stride=8, y_stride=8)
    f.update(kw)
    ptrs = list(ptrs or [P] * 10)
    if at is not None:
        ptrs[at] = ptr
    return ssc.lib().sscater_norm(ctypes.byref(E.NormSpec(*f.values())), *ptrs, None)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(rows=1 << 37), dict(rows=1 << 36, width=1 << 20), dict(width=0), dict(dtype=2),
                                dict(center=2), dict(block_norm=-1), dict(activation=1), dict(activation=2), dict(activation=5),
                                dict(eps=-1.0), dict(eps=float("nan")), dict(x_stride=7), dict(block_stride=7),
                                dict(gate_stride=7), dict(sum_stride=7), dict(y_stride=7), dict(gate_rows=0), dict(gate_rows=3),
                                dict(block_norm=0)])
def test_norm_refuses(kw):
    assert _norm(**kw) == ssc.E_INVALID_ARG


@pytest.mark.parametrize("at", range(10))
def test_norm_refuses_pointers_between_elements(at):
    assert _norm(at, ODD) == ssc.E_INVALID_ARG


def test_norm_refuses_missing_operands():
    assert _norm(1, None) == ssc.E_INVALID_ARG                                        # no block
    assert _norm(9, None) == ssc.E_INVALID_ARG                                        # a weight for a y that is not there
    assert _norm(ptrs=[P, P, P, P, P, P, None, None, None, None]) == ssc.E_INVALID_ARG  # nothing to write
    assert _norm(ptrs=[None] * 8 + [P, P], rows=0) == ssc.OK
    assert ssc.lib().sscater_norm(None, *[P] * 10, None) == ssc.E_INVALID_ARG


def test_linear_takes_no_gate_activation():
    spec = E.LinearSpec(4, 8, 8, E.F32, 4, 8, 8, 8, 8)
    assert ssc.lib().sscater_linear(ctypes.byref(spec), P, P, P, P, P, None) == ssc.E_INVALID_ARG


def _cross(at=None, ptr=None, size=1 << 40, workspace=P, **kw):
    f = dict(dtype=E.BF16, batch=2, q_heads=4, kv_heads=2, head_dim=64, queries=8, keys=20, max_q=4, max_k=10, scale=0.1,
             q_stride=256, k_stride=128, v_stride=128, q_start=None, k_start=None)
    f.update(kw)
    spec = E.CrossSpec(*f.values())
    ptrs = [P] * 5
    if at is not None:
        ptrs[at] = ptr
    rc = ssc.lib().sscater_cross_attend(ctypes.byref(spec), *ptrs, workspace, size, None)
    return rc, ssc.lib().sscater_cross_workspace(ctypes.byref(spec), 1, ctypes.byref(ctypes.c_size_t()))


BAD_CROSS = [dict(dtype=2), dict(batch=0), dict(batch=(1 << 24) + 1), dict(q_heads=0), dict(q_heads=3), dict(kv_heads=0),
             dict(q_heads=(1 << 16) + 2), dict(head_dim=48), dict(queries=-1), dict(queries=9), dict(keys=-1), dict(keys=19),
             dict(max_q=-1), dict(max_q=3), dict(max_k=9), dict(max_q=9, q_start=P, k_start=P),
             dict(max_k=21, q_start=P, k_start=P), dict(q_start=P), dict(k_start=P), dict(q_start=ODD, k_start=P),
             dict(q_start=P, k_start=ODD), dict(scale=float("nan")), dict(q_stride=255), dict(k_stride=127), dict(v_stride=127),
             dict(q_stride=260), dict(k_stride=132), dict(v_stride=132), dict(q_stride=1 << 25), dict(k_stride=1 << 25),
             dict(v_stride=1 << 25), dict(queries=1 << 30, max_q=1 << 30, batch=1, keys=10),
             dict(q_heads=1 << 15, kv_heads=1, q_stride=1 << 21, queries=1 << 17, max_q=1 << 16)]


@pytest.mark.parametrize("kw", BAD_CROSS)
def test_cross_refuses(kw):
    assert _cross(**kw) == (ssc.E_INVALID_ARG, ssc.E_INVALID_ARG)


@pytest.mark.parametrize("at,ptr", [(0, None), (1, None), (2, None), (4, None), (0, OFF), (1, OFF), (2, OFF), (4, OFF)])
def test_cross_refuses_pointers(at, ptr):
    assert _cross(at, ptr)[0] == ssc.E_INVALID_ARG


def test_cross_refuses_a_small_workspace():
    spec = E.CrossSpec(E.F32, 1, 8, 8, 64, 1, 100000, 1, 100000, 0.1, 512, 512, 512, None, None)
    need = ctypes.c_size_t()
    for masked in (0, 1):
        assert ssc.lib().sscater_cross_workspace(ctypes.byref(spec), masked, ctypes.byref(need)) == ssc.OK and need.value > 0
        args = (P, P, P, P if masked else None, P)
        for ptr, size in ((P, need.value - 1), (None, need.value), (OFF, need.value)):
            assert ssc.lib().sscater_cross_attend(ctypes.byref(spec), *args, ptr, size, None) == ssc.E_INVALID_ARG
    assert ssc.lib().sscater_cross_workspace(ctypes.byref(spec), 2, ctypes.byref(need)) == ssc.E_INVALID_ARG
    assert ssc.lib().sscater_cross_workspace(ctypes.byref(spec), 0, None) == ssc.E_INVALID_ARG
    assert ssc.lib().sscater_cross_attend(None, *args, P, 1, None) == ssc.E_INVALID_ARG


def test_rows_behind_the_last_sequence_need_no_workspace():
    need = ctypes.c_size_t()
    for queries, keys in ((4, 9000), (1 << 30, 9000), (4, 1 << 30), (1 << 30, 1 << 30)):
        spec = E.CrossSpec(E.F32, 2, 8, 8, 64, queries, keys, 2, 4500, 0.1, 512, 512, 512, P, P)
        assert ssc.lib().sscater_cross_workspace(ctypes.byref(spec), 1, ctypes.byref(need)) == ssc.OK
        assert need.value < 64 * 4 * 8 * 66 * 4 + (9000 + 2) * 4 + 16
    m, s = E.DeltaMemorySpec(E.F32, 2, 4, 4, 64, 64, P), E.DeltaSpec(1, 1e-6, 0.1, 256, 256, 256, 4, 4)
    sizes = []
    for tokens in (1000, 1 << 30):
        rows = E.TokenRows(tokens, 500, 0, P)
        assert ssc.lib().sscater_delta_workspace(ctypes.byref(s), ctypes.byref(m), ctypes.byref(rows), ctypes.byref(need)) == ssc.OK
        sizes.append(need.value)
    assert sizes[0] == sizes[1] > 0


def test_cross_without_queries_does_nothing():
    assert _cross(queries=0, max_q=0)[0] == ssc.OK


def _delta(at=None, ptr=None, memory=None, rows=None, initial=None, gates=(P, P), **kw):
    m = dict(dtype=E.BF16, batch=2, heads=4, qk_heads=2, key_dim=32, value_dim=64, state=P)
    m.update(memory or {})
    r = dict(tokens=8, max_new=4, max_past=0, start=None)
    r.update(rows or {})
    s = dict(unit=1, eps=1e-6, scale=0.1, q_stride=64, k_stride=64, v_stride=256, a_stride=4, b_stride=4)
    s.update(kw)
    ptrs = [P] * 5
    out = P
    if at is not None and at < 5:
        ptrs[at] = ptr
    elif at is not None:
        out = ptr
    spec, mem, row = E.DeltaSpec(*s.values()), E.DeltaMemorySpec(*m.values()), E.TokenRows(*r.values())
    rc = ssc.lib().sscater_delta_update(ctypes.byref(spec), ctypes.byref(mem), ctypes.byref(row), initial, *ptrs, *gates, out,
                                        P, 1 << 40, None)
    return rc, ssc.lib().sscater_delta_workspace(ctypes.byref(spec), ctypes.byref(mem), ctypes.byref(row),
                                                 ctypes.byref(ctypes.c_size_t()))


BAD = (ssc.E_INVALID_ARG, ssc.E_INVALID_ARG)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(batch=0), dict(batch=(1 << 24) + 1), dict(heads=0), dict(heads=(1 << 16) + 2),
                                dict(qk_heads=0), dict(qk_heads=3), dict(key_dim=48), dict(value_dim=256), dict(state=None),
                                dict(state=OFF)])
def test_delta_refuses_bad_memories(kw):
    assert _delta(memory=kw) == BAD


@pytest.mark.parametrize("kw", [dict(tokens=-1), dict(max_new=-1), dict(max_new=0), dict(max_new=3), dict(max_new=9),
                                dict(max_new=9, start=P), dict(start=ODD), dict(tokens=(1 << 30) + 2, max_new=(1 << 29) + 1)])
def test_delta_refuses_bad_rows(kw):
    assert _delta(rows=kw) == BAD


@pytest.mark.parametrize("kw", [dict(unit=2), dict(eps=-1.0), dict(eps=float("nan")), dict(scale=float("nan")), dict(q_stride=63),
                                dict(k_stride=63), dict(v_stride=255), dict(a_stride=3), dict(b_stride=3)])
def test_delta_refuses_bad_specs(kw):
    assert _delta(**kw) == BAD


@pytest.mark.parametrize("at", range(6))
def test_delta_refuses_pointers(at):
    assert _delta(at, None)[0] == ssc.E_INVALID_ARG
    assert _delta(at, ODD)[0] == ssc.E_INVALID_ARG


def test_delta_refuses_half_of_the_gates():
    assert _delta(gates=(P, None))[0] == ssc.E_INVALID_ARG and _delta(gates=(None, P))[0] == ssc.E_INVALID_ARG
    assert _delta(gates=(ODD, P))[0] == ssc.E_INVALID_ARG and _delta(initial=OFF)[0] == ssc.E_INVALID_ARG


def test_delta_without_tokens_does_nothing():
    none = dict(tokens=0, max_new=0)
    assert _delta(rows=none)[0] == ssc.OK and _delta(rows=none, initial=P)[0] == ssc.OK
