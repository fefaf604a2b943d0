"""Limits of the server's operators that the host checks before any device call: they need no GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2003_10579_b200 import binding
    return binding


@pytest.mark.parametrize("eps", [2.0 ** -127, 2.0 ** 125 * 1.001, 2.0 ** 127, 1e300])
def test_adamw_refuses_eps_whose_reciprocal_is_no_normal_number(B, eps):
    """Divisors over 2^126 have a subnormal reciprocal, which the kernels' division gives as zero: the step would not move."""
    t, h, fake = B.SimAdamwTensor(), C.c_void_p(), 0x10000      # p, m and v in one place: an eps that passes meets the check of overlaps
    ptrs = (C.c_void_p * 1)(fake)
    t.n, t.p, t.m, t.v, t.g = 4, fake, fake, fake, C.cast(ptrs, C.POINTER(C.c_void_p))

    def create(e):
        return B.lib.sim_adamw_create(C.byref(t), 1, 1, 32, 0.9, 0.999, e, 0, C.byref(h))

    assert create(eps) == 1 and b"eps" in B.lib.sim_last_error(None)
    for good in (2.0 ** -126, 1e-8, 2.0 ** 125):
        assert create(good) == 1 and b"overlaps" in B.lib.sim_last_error(None)
