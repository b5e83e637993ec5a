"""Host-side limits of the norms' sizes: calls beyond them are refused before any HIP
work, so the pointers here are never dereferenced."""
import ctypes

import pytest

import paper_2512_08557_amd as ssc
from paper_2512_08557_amd import engine as E

P = ctypes.c_void_p(1 << 20)


@pytest.mark.parametrize("rows,width", [(1 << 36, (1 << 4) + 1), ((1 << 10) + 1, 1 << 30), ((1 << 20) + 1, 1 << 20), ((1 << 36) + 1, 1),
                                        (1, (1 << 30) + 1), (1 << 36, 1 << 28), (1 << 36, (1 << 28) + 16), (1 << 35, 1 << 29),
                                        (1 << 34, 1 << 30), (1 << 36, 1 << 30)])
def test_more_values_than_any_memory_holds(rows, width):
    """Products of 2^64 and more among them."""
    for dtype in (E.F32, E.BF16):
        spec = E.NormSpec(rows, 1, width, dtype, 0, 1, 0, 1e-6, width, width, width, width, width)
        assert ssc.lib().sscater_norm(ctypes.byref(spec), *[P] * 10, None) == ssc.E_INVALID_ARG
