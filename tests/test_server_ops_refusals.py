"""What the server's operators refuse is found on the host before any device call, so it can be checked without a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2003_10579_b200 import binding
    return binding


def _tensor(B, **kw):
    t = B.SimAdamwTensor()
    t.n, t.p_type, t.g_type, t.weight_decay = 64, 0, 0, 0.0
    fake = 0x10000                      # never dereferenced: every case below fails validation first
    t.p = t.m = t.v = t.m_scale = t.v_scale = fake
    ptrs = (C.c_void_p * 2)(fake, fake)
    t.g = C.cast(ptrs, C.POINTER(C.c_void_p))
    t._ptrs = ptrs
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def test_adamw_create_refuses_bad_arguments(B):
    h = C.c_void_p()

    def create(t, n_grads=2, bits=32, b1=0.9, b2=0.999, eps=1e-8, n=1):
        return B.lib.sim_adamw_create(C.byref(t) if t is not None else None, n, n_grads, bits, b1, b2, eps, 0, C.byref(h))

    good = _tensor(B)
    assert create(None) == 1 and create(good, n=0) == 1
    assert create(good, n_grads=0) == 1 and create(good, n_grads=129) == 1
    assert create(good, bits=16) == 1 and b"state_bits" in B.lib.sim_last_error(None)
    for b in (1.0, -0.1, float("nan")):
        assert create(good, b1=b) == 1 and create(good, b2=b) == 1
    for e in (0.0, -1.0, float("nan"), float("inf"), 1e-60):
        assert create(good, eps=e) == 1
    for kw in (dict(n=-1), dict(n=(1 << 40) + 1), dict(p_type=2), dict(p_type=3), dict(g_type=4), dict(g_type=-1), dict(weight_decay=-1.0),
               dict(weight_decay=float("nan")), dict(p=None), dict(m=None), dict(v=None), dict(g=None), dict(p=0x10002), dict(m=0x10001),
               dict(g_type=3), dict(p_type=1, shadow=0x10000)):
        assert create(_tensor(B, **kw)) == 1, kw
        assert not h.value
    assert create(_tensor(B, m_scale=None), bits=8) == 1 and b"m_scale" in B.lib.sim_last_error(None)
    odd = (C.c_void_p * 2)(0x10000, 0x10002)
    assert create(_tensor(B, g=C.cast(odd, C.POINTER(C.c_void_p)))) == 1
    assert B.lib.sim_adamw_create(C.byref(good), 1, 1, 32, 0.9, 0.999, 1e-8, 0, None) == 1


def test_adamw_step_refuses_a_missing_handle(B):
    assert B.lib.sim_adamw_step(None, 1, 1e-3, 1.0, 1, None) == 1
    assert B.lib.sim_adamw_step_device(None, None, None, 1.0, 1, None) == 1
    B.lib.sim_adamw_destroy(None)


def test_adamw_binding_checks_tensors_before_the_library_sees_them(B):
    import torch
    with pytest.raises(ValueError):
        B.AdamW([torch.zeros(4)], [[torch.zeros(4)]])          # CPU tensors
    with pytest.raises(ValueError):
        B.AdamW([], [])
    with pytest.raises(ValueError):
        B.MxTensor(torch.zeros(64, dtype=torch.uint8), torch.zeros(4, dtype=torch.uint8), 1, 128, "linear")
