"""Host-side argument checks of the token operators: every bad call is refused
before any HIP work, so the pointers here are never dereferenced."""
import ctypes

import pytest

import paper_2512_08557_amd as ssc
from paper_2512_08557_amd import engine as E

P = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 1)


def _linear(ptrs=(P, P, P, P, P), **kw):
    f = dict(rows=4, cin=8, cout=8, dtype=E.F32, activation=0, x_stride=8, w_stride=8, residual_stride=8, y_stride=8)
    f.update(kw)
    return ssc.lib().sscater_linear(ctypes.byref(E.LinearSpec(*f.values())), *ptrs, None)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(cin=0), dict(cout=0), dict(dtype=2), dict(activation=4),
                                dict(activation=-1), dict(x_stride=7), dict(w_stride=7), dict(y_stride=7),
                                dict(residual_stride=7), dict(rows=1 << 40), dict(rows=1 << 36, cout=8)])
def test_linear_refuses(kw):
    if kw.get("rows") == 1 << 36:
        kw = dict(kw, cout=1 << 20, y_stride=1 << 20, residual_stride=1 << 20)     # more tiles than a grid takes
    assert _linear(**kw) == ssc.E_INVALID_ARG


@pytest.mark.parametrize("at", [0, 1, 4])
def test_linear_refuses_null_operands(at):
    ptrs = [P] * 5
    ptrs[at] = None
    assert _linear(ptrs) == ssc.E_INVALID_ARG


@pytest.mark.parametrize("at", range(5))
def test_linear_refuses_pointers_between_elements(at):
    ptrs = [P] * 5
    ptrs[at] = ODD
    assert _linear(ptrs) == ssc.E_INVALID_ARG


def test_linear_without_rows_does_nothing():
    assert _linear((None,) * 5, rows=0) == ssc.OK
    assert ssc.lib().sscater_linear(None, P, P, P, P, P, None) == ssc.E_INVALID_ARG


def _cache(**kw):
    f = dict(dtype=E.BF16, batch=2, kv_heads=2, head_dim=64, sinks=4, capacity=100, k=P, v=P, past=P)
    f.update(kw)
    return E.TokenCacheSpec(*f.values())


def _rows(**kw):
    f = dict(tokens=8, max_new=4, max_past=50, start=None)
    f.update(kw)
    return E.TokenRows(*f.values())


BAD_CACHE = [dict(dtype=2), dict(batch=0), dict(kv_heads=0), dict(head_dim=48), dict(sinks=-1), dict(capacity=4),
             dict(capacity=(1 << 30) + 1), dict(k=None), dict(v=None), dict(past=None), dict(k=ODD), dict(v=ODD),
             dict(past=ctypes.c_void_p((1 << 20) + 4))]
BAD_ROWS = [dict(tokens=-1), dict(max_new=-1), dict(max_new=0), dict(max_new=9), dict(max_new=3), dict(max_past=-1),
            dict(max_new=3, start=P), dict(start=ODD)]


def _append(cache, rows, ptrs=(P,) * 6, **kw):
    f = dict(q_heads=4, axes=3, section=(16, 8, 8), interleaved=0, eps=1e-6, qkv_stride=512)
    f.update(kw)
    f["section"] = (ctypes.c_int32 * 3)(*f["section"])
    return ssc.lib().sscater_tokens_append(ctypes.byref(E.HeadSpec(*f.values())), ctypes.byref(cache),
                                           ctypes.byref(rows), *ptrs, None)


def _attend(cache, rows, ptrs=(P, P, P), size=1 << 30, **kw):
    f = dict(q_heads=4, window=16, causal=1, scale=0.125)
    f.update(kw)
    return ssc.lib().sscater_tokens_attend(ctypes.byref(E.AttendSpec(*f.values())), ctypes.byref(cache),
                                           ctypes.byref(rows), ptrs[0], ptrs[1], ptrs[2], size, None)


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_calls_refuse_bad_caches(kw):
    assert _append(_cache(**kw), _rows()) == ssc.E_INVALID_ARG
    assert _attend(_cache(**kw), _rows()) == ssc.E_INVALID_ARG
    assert ssc.lib().sscater_tokens_advance(ctypes.byref(_cache(**kw)), ctypes.byref(_rows()), None) == \
        ssc.E_INVALID_ARG


@pytest.mark.parametrize("kw", BAD_ROWS)
def test_calls_refuse_bad_rows(kw):
    assert _append(_cache(), _rows(**kw)) == ssc.E_INVALID_ARG
    assert _attend(_cache(), _rows(**kw)) == ssc.E_INVALID_ARG
    assert ssc.lib().sscater_tokens_advance(ctypes.byref(_cache()), ctypes.byref(_rows(**kw)), None) == \
        ssc.E_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q_heads=0), dict(axes=0), dict(axes=4), dict(section=(16, 8, 7)),
                                dict(section=(40, -8, 0)), dict(axes=2), dict(interleaved=2), dict(eps=-1.0),
                                dict(eps=float("nan")), dict(qkv_stride=511)])
def test_append_refuses(kw):
    assert _append(_cache(), _rows(), **kw) == ssc.E_INVALID_ARG


@pytest.mark.parametrize("at", [0, 1, 2, 3, 4, 5])
def test_append_refuses_missing_operands(at):
    """qkv, one weight of the two, inv_freq, pos and q."""
    ptrs = [P] * 6
    ptrs[at] = None
    assert _append(_cache(), _rows(), ptrs) == ssc.E_INVALID_ARG
    ptrs[at] = ODD
    assert _append(_cache(), _rows(), ptrs) == ssc.E_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(q_heads=0), dict(q_heads=3), dict(window=0), dict(causal=2),
                                dict(scale=float("nan"))])
def test_attend_refuses(kw):
    assert _attend(_cache(), _rows(), **kw) == ssc.E_INVALID_ARG
    n = ctypes.c_size_t()
    f = dict(q_heads=4, window=16, causal=1, scale=0.125)
    f.update(kw)
    assert ssc.lib().sscater_tokens_workspace(ctypes.byref(E.AttendSpec(*f.values())), ctypes.byref(_cache()),
                                              ctypes.byref(_rows()), ctypes.byref(n)) == ssc.E_INVALID_ARG


def test_attend_refuses_a_cache_that_no_longer_holds_the_reach():
    # 96 ring slots: a window of 93 and four new tokens need exactly those
    need = ctypes.c_size_t()

    def size(window, **kw):
        return ssc.lib().sscater_tokens_workspace(ctypes.byref(E.AttendSpec(4, window, 1, 0.125)),
                                                  ctypes.byref(_cache()), ctypes.byref(_rows(**kw)),
                                                  ctypes.byref(need))
    assert size(93, max_past=1 << 40) == ssc.OK
    assert size(94, max_past=1 << 40) == ssc.E_INVALID_ARG
    # a stream that has not seen more than the ring holds may look back over all of it
    assert size(1 << 30, max_past=92) == ssc.OK
    assert size(1 << 30, max_past=93) == ssc.E_INVALID_ARG


def test_attend_refuses_operands_and_workspace():
    for ptrs in ((None, P, P), (P, None, P), (ODD, P, P), (P, ODD, P)):
        assert _attend(_cache(), _rows(), ptrs) == ssc.E_INVALID_ARG
    n = ctypes.c_size_t()
    big = _cache(capacity=100000)
    rows = _rows(max_past=1 << 40)
    spec = E.AttendSpec(4, 65536, 1, 0.125)
    assert ssc.lib().sscater_tokens_workspace(ctypes.byref(spec), ctypes.byref(big), ctypes.byref(rows),
                                              ctypes.byref(n)) == ssc.OK
    assert n.value > 0                              # few rows over many keys: split
    assert _attend(big, rows, (P, P, P), n.value - 1, window=65536) == ssc.E_INVALID_ARG
    assert _attend(big, rows, (P, P, None), n.value, window=65536) == ssc.E_INVALID_ARG
    assert _attend(big, rows, (P, P, ODD), n.value, window=65536) == ssc.E_INVALID_ARG


def test_calls_without_tokens_do_nothing():
    rows = _rows(tokens=0, max_new=0)
    assert _append(_cache(), rows, (None,) * 6) == ssc.OK
    assert _attend(_cache(), rows, (None, None, None), 0) == ssc.OK
    assert ssc.lib().sscater_tokens_advance(ctypes.byref(_cache()), ctypes.byref(rows), None) == ssc.OK


def test_python_refusals():
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(2, 8), torch.zeros(8, 8)
    with pytest.raises(ValueError, match="cuda"):
        ssc.linear(x, w)
    with pytest.raises(ValueError, match="activation"):
        ssc.linear(x, w, activation="tanh")
    with pytest.raises(ValueError, match="float32"):
        ssc.linear(x.double(), w.double())
    for args, kw in (((1, 1, 48, 8), {}), ((0, 1, 64, 8), {}), ((1, 1, 64, 4), dict(sinks=4)),
                     ((1, 1, 64, 8), dict(dtype="f16"))):
        with pytest.raises(ValueError):
            ssc.TokenCache(*args, **kw)
    with pytest.raises(ValueError, match="axes"):
        ssc.Rotary(None, (8, 8, 8, 8), device="cpu")


@pytest.mark.parametrize("cout,cin", [(3, 0), (0, 8), (0, 0)])
def test_python_linear_refuses_layers_without_channels(cout, cin):
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="at least one channel"):
        ssc.linear(torch.zeros(2, cin), torch.zeros(cout, cin))
