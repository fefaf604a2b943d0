"""What a worker's operators refuse is found on the host before any device call, so it can be checked without a GPU."""
import ctypes as C

import pytest
import torch

F = 0x100000                      # never dereferenced: every case below fails validation first


@pytest.fixture(scope="module")
def B():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2003_10579_b200 import binding
    return binding


def test_checkpoint_calls(B):
    L = B.lib
    assert L.sim_ckpt_codes_bytes(3, 33) == 3 * 64 and L.sim_ckpt_scales_bytes(3, 33) == 6 and L.sim_ckpt_codes_bytes(0, 5) == 0 and L.sim_ckpt_scales_bytes(5, -1) == 0

    def write(x=F, type=1, rows=4, cols=64, ld=64, codes=F * 2, scales=F * 3):
        return L.sim_ckpt_write(x, type, rows, cols, ld, codes, scales, None)

    for kw in (dict(x=None), dict(x=F + 1), dict(type=3), dict(type=-1), dict(rows=-1), dict(cols=-1), dict(cols=1 << 32, ld=1 << 32), dict(ld=63), dict(codes=None), dict(scales=None),
               dict(codes=F * 2 + 8), dict(codes=F + 64), dict(scales=F * 2), dict(scales=F)):
        assert write(**kw) == 1 and b"sim_ckpt_write" in L.sim_last_error(None), kw
    assert write(rows=0, x=None) == 0 and write(cols=0, ld=0) == 0

    def read(codes=F, scales=F * 2, rows=4, cols=64, act=0, type=1, out=F * 3, ld=64):
        return L.sim_ckpt_read(codes, scales, rows, cols, act, type, out, ld, None)

    for kw in (dict(codes=None), dict(scales=None), dict(out=None), dict(out=F * 3 + 1), dict(codes=F + 4), dict(act=4), dict(act=-1), dict(type=3), dict(ld=63), dict(rows=-1), dict(out=F), dict(out=F * 2)):
        assert read(**kw) == 1 and b"sim_ckpt_read" in L.sim_last_error(None), kw
    assert read(rows=0, out=None) == 0


def test_act_backward(B):
    L = B.lib
    room = L.sim_act_backward_workspace(1000, 64)
    assert room > 0 and L.sim_act_backward_workspace(0, 5) == 0

    def call(dy=F, type=1, rows=1000, cols=64, ld=64, codes=F * 2, scales=F * 3, act=2, dz=F * 4, lddz=64, db=F * 5, db_type=0, ws=F * 6, n=room):
        return L.sim_act_backward(dy, type, rows, cols, ld, codes, scales, act, dz, lddz, db, db_type, ws, n, None)

    for kw in (dict(dy=None), dict(dy=F + 1), dict(type=3), dict(rows=-1), dict(ld=63), dict(lddz=63), dict(codes=None), dict(scales=None), dict(dz=None), dict(dz=F * 4 + 1), dict(act=9),
               dict(db_type=3), dict(db=F * 5 + 2), dict(ws=None), dict(n=room - 1), dict(ws=F * 6 + 2), dict(dz=F + 2), dict(dz=F, lddz=65), dict(dz=F * 2), dict(db=F), dict(db=F * 4), dict(ws=F * 4),
               dict(codes=F * 2 + 4), dict(codes=None, scales=None, dz=None, db=None)):
        assert call(**kw) == 1 and b"sim_act_backward" in L.sim_last_error(None), kw


def product(B, **kw):
    p = B.SimProduct(64, 48, 32, 1, F, 32, 0, F * 2, 32, 0, None, 0, 0, 0, None, None, None, 0, F * 3, 1, 48)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def test_matmul(B):
    L = B.lib

    def call(ws=None, n=0, **kw):
        p = product(B, **kw)
        return L.sim_matmul(C.byref(p), ws, n, None)

    for kw in (dict(M=-1), dict(N=-1), dict(K=-1), dict(K=(1 << 30) + 1), dict(type=0), dict(type=3), dict(c_type=2), dict(c_type=3), dict(bias=F * 5, bias_type=2), dict(bias=F * 5 + 2, bias_type=0),
               dict(act=4), dict(act=-1), dict(z_codes=F * 6), dict(z_scales=F * 6), dict(act_grad=1), dict(act_grad=1, z_codes=F * 6, z_scales=F * 7, bias=F * 5, bias_type=1), dict(a=None), dict(b=None),
               dict(a=F + 1), dict(b=F * 2 + 1), dict(lda=31), dict(ldb=31), dict(a_t=1), dict(b_t=1), dict(c=None), dict(c=F * 3 + 1), dict(ldc=47), dict(residual=F * 4, ldr=47), dict(residual=F * 4 + 1, ldr=48),
               dict(z_codes=F * 6 + 8, z_scales=F * 7), dict(c=F), dict(c=F * 2 + 2), dict(residual=F * 3, ldr=50), dict(residual=F * 3 + 2, ldr=48), dict(z_codes=F * 3, z_scales=F * 7),
               dict(z_codes=F, z_scales=F * 7), dict(z_codes=F * 6, z_scales=F * 6), dict(bias=F * 3, bias_type=0)):
        assert call(**kw) == 1 and b"sim_matmul" in L.sim_last_error(None), kw
    assert L.sim_matmul(None, None, 0, None) == 1
    # rows off 16-byte boundaries: room is needed, and has to be apart
    p = product(B, lda=33)
    room = L.sim_matmul_workspace(C.byref(p))
    assert room == 64 * 32 * 2 and L.sim_matmul_workspace(C.byref(product(B))) == 0
    assert call(lda=33) == 1 and call(F * 9, room - 1, lda=33) == 1 and call(F * 9 + 16, room, lda=33) == 1 and call(F * 3, room, lda=33) == 1 and b"workspace" in L.sim_last_error(None)
    assert call(M=0, c=None) == 0 and call(N=0, b=None) == 0


def test_columns_of_one_buffer_do_not_overlap(B):
    """c in columns beside a's (or behind, or wrapped into the next row's start) is no overlap, one element more is.  Nothing is launched: the calls that pass this
    check fail the one of the workspace."""
    L = B.lib

    def call(c, N, ldc=100, lda=100):
        p = product(B, a=F, lda=lda, c=c, ldc=ldc, N=N, b=F * 2 + 2, ldb=33)
        assert L.sim_matmul(C.byref(p), None, 0, None) == 1
        return b"workspace" in L.sim_last_error(None)

    assert call(F + 64, 48) and call(F + 64, 68) and not call(F + 62, 48) and not call(F + 64, 69)
    assert call(F - 200 * 3 + 64, 68) and not call(F - 200 * 3 + 64, 69) and not call(F - 2, 5) and call(F - 10, 5)
    assert not call(F + 64, 48, ldc=104) and not call(F + 64, 48, lda=104)


def test_spans_of_tensors(B):
    buf = torch.zeros(5, 100, dtype=torch.bfloat16)
    ok, bad = ((buf[:, :32], buf[:, 32:80]), (buf[:, 32:], buf[:, :32]), (buf[:2], buf[2:]), (buf[0], buf[1]), (buf.t()[:32], buf[:, 32:]), (buf[:1, 3:4], buf[:, 4:])), (
        (buf[:, :33], buf[:, 32:80]), (buf[:, 32:], buf[:, :33]), (buf[:3], buf[2:]), (buf, buf), (buf.t()[:33], buf[:, 32:]), (buf[0, :5], buf[0, 4:]))
    for a, b in ok:
        B._apart(a, [None, b], "a")
        B._apart(b, [a], "b")
    for a, b in bad:
        for u, v in ((a, b), (b, a)):
            with pytest.raises(ValueError):
                B._apart(u, [v], "u")


def test_the_binding_counts_a_products_room_as_the_library_does(B):
    for a, lda, a_t, b, ldb, b_t in ((F, 32, 0, F * 2, 32, 0), (F + 2, 32, 0, F * 2, 32, 0), (F, 33, 0, F * 2 + 8, 40, 0), (F, 64, 1, F * 2, 49, 1), (F, 71, 1, F * 2, 56, 1)):
        p = product(B, a=a, lda=lda, a_t=a_t, b=b, ldb=ldb, b_t=b_t, c=F * 3)
        assert B.lib.sim_matmul_workspace(C.byref(p)) == B._room(a, lda, a_t, 64, 32) + B._room(b, ldb, b_t, 48, 32)
    one = product(B, M=1, lda=32, a=F, K=31, b=F * 2, ldb=31)
    assert B.lib.sim_matmul_workspace(C.byref(one)) == B._room(F, 32, 0, 1, 31) + B._room(F * 2, 31, 0, 48, 31) > 0


def test_log_probs(B):
    L = B.lib

    def call(x=F, type=1, rows=4, vocab=64, ld=64, tok=F * 2, tb=8, T=1.0, top=2, logp=F * 3, ent=F * 4, lse=F * 5, ids=F * 6, tl=F * 7, g=F * 8, h=F * 9, d=F * 10, ldd=64):
        return L.sim_log_probs(x, type, rows, vocab, ld, tok, tb, T, top, logp, ent, lse, ids, tl, g, h, d, ldd, None)

    for kw in (dict(x=None), dict(x=F + 1), dict(type=3), dict(rows=-1), dict(rows=1 << 28), dict(vocab=0), dict(vocab=(1 << 30) + 1, ld=1 << 31), dict(ld=63), dict(ldd=63), dict(T=0.0), dict(T=-1.0),
               dict(T=float("nan")), dict(T=float("inf")), dict(top=-1), dict(top=33), dict(top=0), dict(top=2, ids=None, tl=None), dict(vocab=1, top=2), dict(tb=2), dict(tok=None), dict(tok=F * 2 + 4),
               dict(d=None), dict(d=F * 10 + 1), dict(logp=F * 3 + 2), dict(d=F + 2), dict(d=F, ldd=65), dict(logp=F), dict(ent=F * 3), dict(ids=F * 7), dict(lse=F * 8), dict(tl=F * 2)):
        assert call(**kw) == 1 and b"sim_log_probs" in L.sim_last_error(None), kw
    assert call(rows=0, x=None) == 0


def test_binding_checks_tensors_before_the_library_sees_them(B):
    import torch
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(3, 8, dtype=torch.bfloat16)
    for call in (lambda: B.checkpoint(x), lambda: B.linear(x, w), lambda: B.linear(x, w, act="tanh"), lambda: B.linear_backward(x, x, w), lambda: B.log_probs(x), lambda: B.log_probs_backward(x, None),
                 lambda: B.act_backward(x, None, "relu"), lambda: B.checkpoint_read(None, act="x"),
                 lambda: B.Checkpoint(torch.zeros(64, dtype=torch.uint8), torch.zeros(4, dtype=torch.uint8), 1, 64)):
        with pytest.raises(ValueError):
            call()
