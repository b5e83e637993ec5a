"""Host-side argument checks of cross attention: every bad call is refused before any
HIP work, so the pointers here are never dereferenced."""
import ctypes

import pytest

import paper_2512_08557_amd as ssc
from paper_2512_08557_amd import engine as E

P = ctypes.c_void_p(1 << 20)


@pytest.mark.parametrize("rounded", [-1, 2])
@pytest.mark.parametrize("dtype", [E.F32, E.BF16])
def test_rounded_is_zero_or_one(dtype, rounded):
    spec = E.CrossSpec(dtype, 1, 8, 8, 64, 40, 100000, 40, 100000, 0.1, 512, 512, 512, None, None, rounded)
    need = ctypes.c_size_t()
    assert ssc.lib().sscater_cross_workspace(ctypes.byref(spec), 0, ctypes.byref(need)) == ssc.E_INVALID_ARG
    assert ssc.lib().sscater_cross_attend(ctypes.byref(spec), P, P, P, None, P, P, 1 << 40, None) == ssc.E_INVALID_ARG
    sizes = []
    for spec.rounded in (0, 1):
        assert ssc.lib().sscater_cross_workspace(ctypes.byref(spec), 0, ctypes.byref(need)) == ssc.OK
        sizes.append(need.value)
    assert sizes[0] == sizes[1]
