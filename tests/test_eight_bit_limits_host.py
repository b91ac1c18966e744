"""CPU tests of the limits of the operators of 8-bit affine blocks: what they refuse at the ends of their ranges."""

import ctypes

import pytest

import paper_2006_03108_b200 as distdl

torch = pytest.importorskip("torch")
vp = ctypes.c_void_p


def test_norm_refuses_eps_whose_squares_are_subnormal():
    """What weighs against an eps of 2^-120 has squares whose error is 2^-30 of it; below, they lose the digits that the sums count on."""
    lib, a = distdl.lib(), (vp * 1)(0x10000)

    def status(eps, nb=0):
        return lib.distdl_rmsnorm_fwd(nb, 128, 1, a, None, a, ctypes.byref(ctypes.c_double(eps)), distdl.F32, a, None, None, None, None, None)

    assert status(2.0 ** -120) == 0 and status(1e-6) == 0 and status(3e38) == 0             # no samples: nothing to do
    for eps in (2.0 ** -120 * (1 - 2.0 ** -50), 2.0 ** -121, 2.0 ** -130, 1e-45, 0.0, -1.0, float("nan"), float("inf"), 1e39):
        assert status(eps) == 1 and status(eps, 4) == 1, eps
        assert b"eps" in lib.distdl_last_error()
