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
    # p, m and v in one place: the step would write them over one another
    assert create(good) == 1 and b"overlaps" in B.lib.sim_last_error(None)
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


def test_mx_calls_refuse_bad_arguments(B):
    L, f = B.lib, 0x10000
    assert L.sim_mx_codes_bytes(3, 129) == 3 * 128 and L.sim_mx_scales_bytes(129, 129, 1) == 4 * 512 and L.sim_mx_scales_bytes(3, 33, 0) == 6
    assert L.sim_mx_codes_bytes(0, 5) == 0 and L.sim_mx_scales_bytes(1 << 30, 1 << 30, 1) == 0

    def quant(x=f, type=0, rows=4, cols=64, ld=64, tiles=1, codes=f, scales=f, codes_t=None, scales_t=None):
        return L.sim_mx_quantize(x, type, rows, cols, ld, tiles, 0, 0, codes, scales, codes_t, scales_t, None)

    for kw in (dict(x=None), dict(x=f + 2), dict(type=3), dict(type=-1), dict(rows=0), dict(cols=0), dict(cols=-5), dict(rows=1 << 36), dict(ld=63), dict(ld=1 << 50),
               dict(codes=None), dict(scales=None), dict(codes=None, scales=None), dict(codes_t=f), dict(scales_t=f), dict(codes=f + 8), dict(scales=f + 4),
               dict(codes_t=f + 8, scales_t=f), dict(codes_t=f, scales_t=f + 8)):
        assert quant(**kw) == 1, kw
        assert b"sim_mx_quantize" in L.sim_last_error(None)

    def read(codes=f, scales=f, rows=4, cols=64, type=0, out=f, ld=64):
        return L.sim_mx_dequantize(codes, scales, rows, cols, 1, type, out, ld, None)

    for kw in (dict(codes=None), dict(scales=None), dict(out=None), dict(out=f + 2), dict(type=3), dict(rows=0), dict(cols=0), dict(ld=63)):
        assert read(**kw) == 1, kw

    def product(a=f, sa=f, b=f, sb=f, M=4, N=4, K=64, type=0, c=f, ldc=4):
        return L.sim_mx_matmul(a, sa, b, sb, M, N, K, type, c, ldc, None)

    for kw in (dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(c=None), dict(c=f + 2), dict(a=f + 8), dict(sb=f + 8), dict(M=0), dict(N=0), dict(K=0),
               dict(K=(1 << 30) + 1), dict(type=2), dict(type=3), dict(ldc=3), dict(M=1 << 30, N=1 << 30, ldc=1 << 30)):
        assert product(**kw) == 1, kw
