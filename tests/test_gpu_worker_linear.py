"""A worker's products with their tails, forward and backward, against 64 bits.

Tolerances.  Both operands are exact in fp32, and so is each product of two elements.  An fp32 sum of K terms in any order is off by at most
K 2^-23 of the sum of magnitudes (2^-24 a step, twice that if the tensor core truncates); bias adds a step.  Activations have a slope of at
most 1.13 and are off by 2^-18 |z| themselves (exponential and reciprocal 2^-21 together, the exponent's rounding the rest).  Their
slopes are off by at most 2^-14: q (1 - q) by 2^-20, times |z| sqrt(8 / pi) (1 + 0.134 z^2) < 2^6 while |z| < 6; beyond, q (1 - q) is
nothing but the rounding 2^-23 of 1 - q, times less than 2^8.  The result adds half a step of its type.  A kept matrix is the rounding of
a value that is itself within the sum's tolerance: within half a step of E4M3 (2^-4 of the value, or 2^-10 of the scale) plus that."""
import itertools

import numpy as np
import pytest
import torch

from worker_ref import EPS, TINY, act, close, f64, keep, slope, values

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def normal(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * scale).to(dtype)


def sum_tol(a, b):
    """Of a b^T with K columns each: K 2^-23 of the sum of magnitudes."""
    return max(1, a.shape[1]) * 2.0**-23 * (np.abs(a) @ np.abs(b).T)


def check_linear(B, x, w, bias=None, a="none", residual=None, keep_z=False, dtype=None, out=None):
    got = B.linear(x, w, bias, act=a, residual=residual, keep=keep_z, dtype=dtype, out=out)
    got, z8 = got if keep_z else (got, None)
    X, W = f64(x).reshape(-1, x.shape[-1]), f64(w)
    z, tol = X @ W.T, sum_tol(X, W)
    if bias is not None:
        z = z + f64(bias)
        tol = tol + 2.0**-23 * np.abs(z)
    want = act(a, z)
    t = 1.13 * tol + 2.0**-18 * np.abs(z) * (a not in ("none", "relu"))
    if residual is not None:
        want = want + f64(residual).reshape(want.shape)
        t = t + 2.0**-23 * (np.abs(want) + np.abs(f64(residual).reshape(want.shape)))
    close(got, want, t * (1 + EPS[got.dtype]) + EPS[got.dtype] * np.abs(want) + TINY[got.dtype], "y")
    if keep_z:
        v, k = values(z8)
        scale = np.repeat(np.exp2(k), 32, 1)[:, : v.shape[1]]
        close(v, z, np.maximum(2.0**-4 * np.abs(z), 2.0**-10 * scale) + 1.07 * tol, "kept")
        pad = -z.shape[1] % 32
        top = np.abs(np.pad(z, ((0, 0), (0, pad)))).reshape(len(z), -1, 32).max(-1)
        slack = np.pad(tol, ((0, 0), (0, pad))).reshape(top.shape + (32,)).max(-1)
        assert (448 * np.exp2(k) >= top - slack).all() and ((224 * np.exp2(k) < top + slack) | (k == -127)).all()
    return got


SHAPES = [(1, 8, 16), (1, 4096, 640), (2, 100, 33), (7, 2051, 515), (16, 64, 128), (17, 72, 200), (33, 520, 1000), (64, 1024, 96), (65, 1024, 130), (100, 40, 31),
          (128, 128, 128), (129, 200, 257), (300, 24, 17), (500, 333, 64), (700, 2048, 48), (1000, 1500, 10), (513, 4200, 513), (1300, 2176, 2000), (2048, 512, 2100)]


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_forward_over_shapes(B, M, K, N):
    gen = torch.Generator(device=DEV).manual_seed(M * 7 + K + N)
    dt = torch.float16 if (M + N) % 3 == 0 else torch.bfloat16
    x, w = normal(gen, M, K, dtype=dt), normal(gen, N, K, dtype=dt, scale=K**-0.5)
    check_linear(B, x, w)
    check_linear(B, x, w, normal(gen, N, dtype=torch.float32), "gelu", normal(gen, M, N, dtype=dt), keep_z=True)
    check_linear(B, x, w, normal(gen, N, dtype=dt), "relu", dtype=torch.float32, keep_z=True)


@pytest.mark.parametrize("a,dt,odt,bt,res", [c for i, c in enumerate(itertools.product(("none", "relu", "gelu", "silu"), (torch.bfloat16, torch.float16), ("same", "f32"), ("same", "f32", None), (True, False))) if i % 3 != 1])
@pytest.mark.parametrize("M,K,N", [(5, 96, 70), (140, 96, 200), (2304, 64, 2304)])
def test_every_tail(B, a, dt, odt, bt, res, M, K, N):
    gen = torch.Generator(device=DEV).manual_seed(11)
    odt = dt if odt == "same" else torch.float32
    bias = None if bt is None else normal(gen, N, dtype=dt if bt == "same" else torch.float32)
    check_linear(B, normal(gen, M, K, dtype=dt), normal(gen, N, K, dtype=dt, scale=0.1), bias, a, normal(gen, M, N, dtype=odt) if res else None, keep_z=res, dtype=odt)


@pytest.mark.parametrize("M,K,N", [(3, 40, 50), (40, 70, 300), (200, 136, 150), (2400, 72, 2300)])
@pytest.mark.parametrize("pad", [0, 1, 3, 8])
def test_strides_and_alignment(B, M, K, N, pad):
    """Rows apart by more than their length, at odd addresses, and the results between guards."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    off = pad % 2

    def framed(t, fill):
        full = torch.full((t.shape[0] * (t.shape[1] + pad) + 16,), fill, dtype=t.dtype, device=DEV)
        v = full[off: off + t.shape[0] * (t.shape[1] + pad)].view(t.shape[0], t.shape[1] + pad)[:, : t.shape[1]]
        v.copy_(t)
        return full, v

    _, x = framed(normal(gen, M, K), 7.0)
    _, w = framed(normal(gen, N, K, scale=0.1), 7.0)
    _, r = framed(normal(gen, M, N), 7.0)
    full, out = framed(torch.zeros(M, N, dtype=torch.bfloat16, device=DEV), 3.0)
    bias = normal(gen, N + 1, dtype=torch.float32)[1:]
    got = check_linear(B, x, w, bias, "silu", r, keep_z=True, out=out)
    assert got.data_ptr() == out.data_ptr()
    seen = torch.zeros(full.numel(), dtype=torch.bool, device=DEV)
    seen[off: off + M * (N + pad)].view(M, N + pad)[:, :N] = True
    assert (full[~seen] == 3.0).all()


def test_operands_in_either_order_and_the_residual_in_place(B):
    gen = torch.Generator(device=DEV).manual_seed(6)
    for M, K, N in [(3, 48, 40), (50, 200, 300), (150, 72, 136), (2312, 136, 2304)]:
        xt, wt = normal(gen, K, M), normal(gen, K, N, scale=0.1)
        r = normal(gen, M, N)
        for x, w in ((xt.t(), wt.t()), (xt.t(), wt.t().contiguous()), (xt.t().contiguous(), wt.t())):
            check_linear(B, x, w, None, "none", r)
        c = r.clone()
        want = B.linear(xt.t(), wt.t(), residual=r)
        got = B.linear(xt.t(), wt.t(), residual=c, out=c)
        assert got is c and torch.equal(got, want)


def test_one_token_as_a_vector_and_nothing_at_all(B):
    gen = torch.Generator(device=DEV).manual_seed(7)
    x, w, bias = normal(gen, 24), normal(gen, 70, 24), normal(gen, 70)
    assert torch.equal(B.linear(x, w, bias), B.linear(x[None], w, bias))
    assert B.linear(x[None][:0], w, bias).shape == (0, 70)
    y, z = B.linear(x[None][:0], w, bias, keep=True)
    assert y.shape == (0, 70) and z.rows == 0 and z.codes.numel() == 0
    assert B.linear(x[None], w[:0]).shape == (1, 0)
    none = torch.zeros(5, 0, dtype=torch.bfloat16, device=DEV)
    y = B.linear(none, torch.zeros(70, 0, dtype=torch.bfloat16, device=DEV), bias, act="silu")
    close(y, np.repeat(act("silu", f64(bias))[None], 5, 0), 2.0**-8 * np.abs(act("silu", f64(bias))) + 2.0**-17, "no k")
    none = torch.zeros(300, 0, dtype=torch.bfloat16, device=DEV)
    assert (B.linear(none, torch.zeros(700, 0, dtype=torch.bfloat16, device=DEV)) == 0).all()
    dx, dw, db = B.linear_backward(torch.zeros(0, 70, dtype=torch.bfloat16, device=DEV), x[None][:0], w)
    assert dx.shape == (0, 24) and (dw == 0).all() and (db == 0).all() and dw.shape == (70, 24)


def test_infinities_and_nan_stay_where_they_are(B):
    gen = torch.Generator(device=DEV).manual_seed(8)
    for M, K, N in [(4, 64, 96), (200, 64, 96), (2304, 64, 2304)]:
        x, w = normal(gen, M, K), normal(gen, N, K)
        x[1, 3], x[2, 5] = float("nan"), float("inf")
        for a in ("none", "relu"):
            y, z = B.linear(x, w, act=a, keep=True)
            bad = ~torch.isfinite(y)
            assert torch.isnan(y[1]).all() and not bad[0].any() and not bad[3:].any()
            v, k = values(z)
            assert np.isnan(v[1:3]).all() and (k[1:3] == 128).all() and np.isfinite(v[0]).all() and np.isfinite(v[3:]).all()


def test_the_same_bits_every_time_and_under_a_graph(B):
    gen = torch.Generator(device=DEV).manual_seed(9)
    for M, K, N in [(1, 4096, 1024), (40, 3001, 700), (300, 8192, 300), (1500, 2048, 1600)]:
        x, w, r = normal(gen, M, K), normal(gen, N, K, scale=0.02), normal(gen, M, N)
        want, z = B.linear(x, w, act="gelu", residual=r, keep=True)
        for _ in range(3):
            y, z2 = B.linear(x, w, act="gelu", residual=r, keep=True)
            assert torch.equal(y, want) and torch.equal(z.codes, z2.codes) and torch.equal(z.scales, z2.scales)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = B.linear(x, w, act="gelu", residual=r)
        y.zero_()
        g.replay()
        assert torch.equal(y, want)
        x.copy_(normal(gen, M, K))
        want2 = B.linear(x, w, act="gelu", residual=r)
        g.replay()
        assert torch.equal(y, want2)


def test_on_another_stream(B):
    gen = torch.Generator(device=DEV).manual_seed(10)
    x, w = normal(gen, 100, 777), normal(gen, 300, 777, scale=0.1)
    want, wz = B.linear(x, w, act="silu", keep=True)
    grads = B.linear_backward(want, B.checkpoint(x), w, x_act="gelu")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    y, z = B.linear(x, w, act="silu", keep=True, stream=st)
    more = B.linear_backward(y, B.checkpoint(x, stream=st), w, x_act="gelu", stream=st)
    st.synchronize()
    assert torch.equal(y, want) and torch.equal(z.codes, wz.codes) and all(torch.equal(a, b) for a, b in zip(grads, more))


@pytest.mark.parametrize("T,fin,fout", [(1, 16, 40), (5, 130, 77), (37, 515, 300), (64, 1024, 1024), (130, 96, 300), (1531, 333, 129), (2300, 2304, 2310), (4, 3000, 8), (9000, 40, 24)])
@pytest.mark.parametrize("a", ["tensor", "none", "relu", "gelu", "silu"])
def test_backward(B, T, fin, fout, a):
    gen = torch.Generator(device=DEV).manual_seed(T + fin)
    dt = torch.float16 if fout % 3 == 0 else torch.bfloat16
    v, dy, w = normal(gen, T, fin, dtype=dt), normal(gen, T, fout, dtype=dt, scale=0.1), normal(gen, fout, fin, dtype=dt, scale=fin**-0.5)
    skip = normal(gen, T, fin, dtype=dt, scale=0.1) if a != "relu" else None
    odt = dt if a == "gelu" else torch.float32
    if a == "tensor":
        x, name, V = v, "none", f64(v)
        H = V
    else:
        x, name = B.checkpoint(v), a
        V = keep(f64(v))[0]
        H = f64(B.checkpoint_read(x, dt, act=a))          # the rounding of x_act(v) to dy's type is part of the definition
        close(H, act(a, V), EPS[dt] * np.abs(act(a, V)) + 2.0**-18 * np.abs(V) + TINY[dt], "h")
    dx, dw, db = B.linear_backward(dy, x, w, x_act=name, residual=skip, dtype=odt)
    G, W = f64(dy), f64(w)
    s, S = slope(name, V), np.abs(slope(name, V))
    want = (G @ W) * s
    tol = sum_tol(G, W.T) * (S + 2.0**-14) + np.abs(G @ W) * 2.0**-14 * (name not in ("none", "relu"))
    if skip is not None:
        want = want + f64(skip)
        tol = tol + 2.0**-23 * (np.abs(want) + np.abs(f64(skip)))
    close(dx, want, tol * (1 + EPS[dt]) + EPS[dt] * np.abs(want) + TINY[dt], "dx")
    want, tol = G.T @ H, sum_tol(G.T, H.T)
    close(dw, want, tol * (1 + EPS[odt]) + EPS[odt] * np.abs(want) + TINY[odt], "dw")
    want, tol = G.sum(0), T * 2.0**-24 * np.abs(G).sum(0)
    close(db, want, tol * (1 + EPS[odt]) + EPS[odt] * np.abs(want) + TINY[odt], "db")
    only = B.linear_backward(dy, x, w, x_act=name, need="w", dtype=odt)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)


def test_backward_against_differences(B):
    """The loss sum(y c) of a two-layer block in 64 bits, moved along single entries: what the three products return is its gradient, up to the
    rounding of the intermediate gradient to 16 bits (2^-8 of each element)."""
    gen = torch.Generator(device=DEV).manual_seed(12)
    T, d, f = 6, 24, 40
    v, w1, w2, c = normal(gen, T, d), normal(gen, f, d, scale=0.3), normal(gen, d, f, scale=0.3), normal(gen, T, d)
    b1 = normal(gen, f, dtype=torch.float32)
    v = B.checkpoint_read(B.checkpoint(v), torch.bfloat16)            # values that 8 bits hold
    z8 = B.linear(v, w1, b1, keep=True)[1]
    dz, dw2, db2 = B.linear_backward(c, z8, w2, x_act="gelu")
    dx, dw1, db1 = B.linear_backward(dz, B.checkpoint(v), w1, residual=c)
    V, W1, W2, C, b = f64(v), f64(w1), f64(w2), f64(c), f64(b1)
    shift = values(z8)[0] - (V @ W1.T + b)                            # the kept z: the block is differentiated there

    def loss(V, W1, W2, b):
        return ((act("gelu", V @ W1.T + b + shift) @ W2.T + V) * C).sum()

    rng = np.random.default_rng(0)
    mag = np.abs(f64(dz))
    h = act("gelu", values(z8)[0])
    for name, got, at, tol in (("dx", dx, 0, mag @ np.abs(W1)), ("dw1", dw1, 1, mag.T @ np.abs(V)), ("dw2", dw2, 2, np.abs(C).T @ np.abs(h)), ("db1", db1, 3, mag.sum(0))):
        args = [V, W1, W2, b]
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in args[at].shape)
            e = 1e-4
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[at][i] += e
            down[at][i] -= e
            want = (loss(*up) - loss(*down)) / (2 * e)
            # rounding of dz or h (2^-8 of each term), of the result, the differences' own error
            assert abs(float(f64(got)[i]) - want) <= 2.0**-8 * tol[i] * 1.01 + 2.0**-8 * abs(want) + 1e-5 * (1 + abs(want)), (name, i)


def test_long_rows_pass_32_bits(B):
    """c has more than 2^31 elements: the last rows are where they belong."""
    gen = torch.Generator(device=DEV).manual_seed(13)
    M, K, N = 70000, 16, 32768
    x, w = normal(gen, M, K), normal(gen, N, K)
    y = B.linear(x, w)
    for r in (0, 65535, 65536, M - 1):
        X, W = f64(x[r:r + 1]), f64(w)
        want = X @ W.T
        close(y[r:r + 1], want, sum_tol(X, W) * 1.01 + 2.0**-8 * np.abs(want), "row %d" % r)
