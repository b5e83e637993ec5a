"""Host-side limits of sizes: calls beyond them are refused before any HIP work,
so the pointers here are never dereferenced."""
import ctypes

import pytest

import paper_2512_08557_amd as ssc
from paper_2512_08557_amd import engine as E

P = ctypes.c_void_p(1 << 20)


@pytest.mark.parametrize("rows,cout", [(1 << 36, (1 << 4) + 1), ((1 << 10) + 1, 1 << 30), ((1 << 20) + 1, 1 << 20),
                                       ((1 << 36) + 1, 1), (1, (1 << 30) + 1), (1 << 36, 1 << 30)])
def test_linear_refuses_more_outputs_than_any_memory_holds(rows, cout):
    for dtype in (E.F32, E.BF16):
        spec = E.LinearSpec(rows, 8, cout, dtype, 0, 8, 8, cout, cout)
        assert ssc.lib().sscater_linear(ctypes.byref(spec), P, P, None, None, P, None) == ssc.E_INVALID_ARG


def test_rows_beyond_limits_are_refused():
    cache = E.TokenCacheSpec(E.BF16, 1, 1, 32, 0, 1 << 30, P, P, P)
    need = ctypes.c_size_t()

    def size(tokens, heads, **kw):
        rows = E.TokenRows(tokens, tokens, kw.get("max_past", 0), None)
        return ssc.lib().sscater_tokens_workspace(ctypes.byref(E.AttendSpec(heads, 1, 1, 1.0)), ctypes.byref(cache),
                                                  ctypes.byref(rows), ctypes.byref(need))
    assert size(1 << 30, 1) == ssc.OK and size(1 << 14, 1 << 16) == ssc.OK and size(1, 1, max_past=1 << 62) == ssc.OK
    assert size((1 << 30) + 1, 1) == size((1 << 14) + 1, 1 << 16) == size(1, (1 << 16) + 1) == ssc.E_INVALID_ARG
    assert size(1, 1, max_past=(1 << 62) + 1) == ssc.E_INVALID_ARG
