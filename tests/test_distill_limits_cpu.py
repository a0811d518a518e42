"""Parameters of the distillation loss whose fp32 form is no number, or 0, are refused.  No kernel
is launched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2609_32444_gb300 import binding as b
    from paper_2609_32444_gb300 import build
    build.build()
    b.lib()
    return b


@pytest.mark.parametrize("name,value", [("coef", 1e39), ("coef", -1e300), ("coef", 1.1e30),
                                        ("tail_min", 1e-46), ("tail_min", 1e-300),
                                        ("tail_min", 9e-31)])
def test_values_outside_fp32(binding, name, value):
    P = binding.cis_distill_default_params(**{name: value})
    z, dz, ws = (ctypes.c_void_p(x) for x in (0x10000, 0x4000000, 0x20000))
    assert binding.lib().cis_distill_fwd_bwd(
        z, 1, 4, 8, 8, z, z, 3, 3, None, None, None, 0, ctypes.byref(P), dz, 1, 8, None, None, ws,
        1 << 20, None) == 1
