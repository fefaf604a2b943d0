"""Activations kept in 8 bits: written, read back through an activation, used for the gradient; against 64 bits.

What is kept has no tolerance: blocks of 32 and E4M3 are arithmetic on the type's exact values.  Reading adds the activation's error
(2^-18 |z|, see the products' tests) and half a step of the type; gradients the slope's (2^-14) and half a step; sums of R rows
R 2^-24 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from worker_ref import EPS, TINY, act, close, f64, in_range, keep, slope, values

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def matrix(rows, cols, dt, seed, pad=0, off=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    full = torch.randn(rows * (cols + pad) + 16, generator=gen, device=DEV).to(dt)
    x = full[off: off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    x *= torch.exp2(torch.randint(-6, 7, (rows, 1), generator=gen, device=DEV).float()).to(dt)
    return x


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,cols,pad,off", [(1, 1, 0, 0), (3, 31, 0, 0), (2, 32, 0, 0), (5, 33, 3, 1), (7, 100, 4, 0), (77, 768, 0, 0), (77, 768, 0, 1), (300, 1001, 0, 0), (1000, 264, 8, 0), (1, 70000, 0, 0)])
def test_write_and_read(B, dt, rows, cols, pad, off):
    x = matrix(rows, cols, dt, rows + cols, pad, off)
    q = B.checkpoint(x)
    want, k, units = keep(f64(x))
    got, gk = values(q)
    assert np.array_equal(gk, k) and np.array_equal(got, want)
    for a in ("none", "relu", "gelu", "silu"):
        for odt in TYPES:
            y = B.checkpoint_read(q, odt, act=a)
            w = act(a, want)
            close(y, w, EPS[odt] * np.abs(w) + TINY[odt] + 2.0**-18 * np.abs(want) * (a in ("gelu", "silu")), a)
    buf = torch.full((rows * (cols + 5) + 3,), 9.0, dtype=torch.bfloat16, device=DEV)
    out = buf[1: 1 + rows * (cols + 5)].view(rows, cols + 5)[:, :cols]
    assert torch.equal(B.checkpoint_read(q, act="gelu", out=out), B.checkpoint_read(q, torch.bfloat16, act="gelu"))
    assert (buf[1: 1 + rows * (cols + 5)].view(rows, cols + 5)[:, cols:] == 9.0).all() and buf[0] == 9.0 and (buf[-2:] == 9.0).all()


def test_ends_of_the_range(B):
    top = torch.finfo(torch.float32).max
    rows = [[0.0] * 40, [top] + [1.0] * 39, [1e-45] * 40, [2.0**-126] * 40, [448.0, 449.0] + [0.0] * 38, [448.0] + [17.0, 18.0, 19.0, 2.0**-10, 3 * 2.0**-10, 2.0**-9] + [-0.0] * 33,
            [float("inf")] + [1.0] * 39, [1.0] * 39 + [float("nan")], [-top] * 40, [2.0**-119] * 40]
    for dt in (torch.float32, torch.bfloat16):
        x = torch.tensor(rows, device=DEV).to(dt)
        for v in (x, torch.cat([x, x], 1)[:, :41][:, 1:]):
            q = B.checkpoint(v)
            want, k, _ = keep(f64(v))
            got, gk = values(q)
            assert np.array_equal(gk, k) and np.array_equal(got, want, equal_nan=True)
            # the largest fp32 number is 255.99 times 2^120: kept as 256, which reads as 2^128, beyond fp32
            close(B.checkpoint_read(q, torch.float32), in_range(want, torch.float32), TINY[torch.float32] + 0 * np.abs(want), "read")
    assert np.isnan(f64(B.checkpoint_read(B.checkpoint(torch.tensor(rows, device=DEV)), act="relu")))[6, :32].all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("a", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,pad,off", [(1, 5, 0, 0), (9, 40, 0, 0), (77, 768, 0, 0), (33, 257, 3, 1), (1500, 520, 8, 0), (1500, 519, 0, 0), (5000, 31, 0, 0)])
def test_gradient_and_its_sums(B, dt, a, rows, cols, pad, off):
    dy, z = matrix(rows, cols, dt, 3 * rows + cols, pad, off), B.checkpoint(matrix(rows, cols, dt, rows - cols, pad, off))
    dz, db = B.act_backward(dy, z, a)
    G, V = f64(dy), values(z)[0]
    want = G * slope(a, V)
    off_by = 2.0**-23 * np.abs(want) + np.abs(G) * 2.0**-14 * (a in ("gelu", "silu"))
    close(dz, want, off_by * 1.01 + EPS[dt] * np.abs(want) + TINY[dt], "dz")
    close(db, want.sum(0), off_by.sum(0) + rows * 2.0**-24 * np.abs(want).sum(0) * 1.01 + TINY[torch.float32], "db")
    assert torch.equal(B.act_backward(dy, z, a)[1], db)
    db16 = B.act_backward(dy, z, a, dtype=torch.bfloat16)[1]
    assert torch.equal(db16, db.to(torch.bfloat16))
    assert B.act_backward(dy, z, a, bias=False)[1] is None
    copy = dy.clone()
    same, _ = B.act_backward(copy, z, a, out=(copy, None))
    assert same is copy and torch.equal(copy, dz)


def test_gradient_against_differences(B):
    z = torch.linspace(-9, 9, 1024, device=DEV)
    q = B.checkpoint(z)
    V, e = values(q)[0], 1e-5
    for a in ("gelu", "silu"):
        dz, _ = B.act_backward(torch.ones(1, 1024, device=DEV), q, a)
        close(dz, (act(a, V + e) - act(a, V - e)) / (2 * e), 2.0**-14 + 1e-8, a)


@pytest.mark.parametrize("cols", [96, 70])
@pytest.mark.parametrize("a", ["none", "relu", "gelu", "silu"])
def test_a_nan_block_stays_one(B, a, cols):
    """The gradient through a block that could not be kept is NaN, its neighbours' is not, and so are the columns' sums."""
    x = matrix(40, cols, torch.bfloat16, 8)
    x[3, 40] = float("inf")
    dy, q = matrix(40, cols, torch.bfloat16, 9), B.checkpoint(x)
    dz, db = B.act_backward(dy, q, a)
    bad = torch.zeros(40, cols, dtype=torch.bool, device=DEV)
    bad[3, 32:64] = True
    assert torch.equal(torch.isnan(dz), bad) and torch.equal(torch.isnan(db), bad.any(0))
    w = matrix(24, cols, torch.bfloat16, 10)
    for rows in (slice(0, 40), slice(0, 4)):
        part = B.Checkpoint(q.codes, q.scales, 40 if rows.stop == 40 else 4, cols)
        dx = B.linear_backward(matrix(40, 24, torch.bfloat16, 11)[rows], part, w, x_act=a, need="x")[0]
        assert torch.equal(torch.isnan(dx), bad[rows]) or a == "none"


def test_nothing(B):
    for rows, cols in ((0, 5), (0, 64)):
        x = torch.zeros(rows, cols, device=DEV)
        q = B.checkpoint(x)
        assert B.checkpoint_read(q).shape == (rows, cols)
        dz, db = B.act_backward(x, q, "gelu")
        assert dz.shape == (rows, cols) and (db == 0).all() and db.numel() == cols


def test_rows_far_apart(B):
    """Offsets beyond 2^31 elements."""
    x = torch.zeros(3, 1 << 30, dtype=torch.bfloat16, device=DEV)
    x[2, 5:40] = torch.arange(35, device=DEV).to(torch.bfloat16)
    v = x[:, :64]
    q = B.checkpoint(v)
    assert np.array_equal(values(q)[0], keep(f64(v))[0])
    dz, db = B.act_backward(v, q, "none")
    assert torch.equal(dz, v) and torch.equal(db, v.float().sum(0))
    del x, v


def test_graph(B):
    x, dy = matrix(500, 300, torch.bfloat16, 1), matrix(500, 300, torch.bfloat16, 2)
    B.act_backward(dy, B.checkpoint(x), "silu")
    graphs = []
    for _ in range(2):          # two graphs, each with room of its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q = B.checkpoint(x)
            out = B.act_backward(dy, q, "silu")
        graphs.append((g, out))
    x.copy_(matrix(500, 300, torch.bfloat16, 3))
    want = B.act_backward(dy, B.checkpoint(x), "silu")
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(5):
        for (g, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


@pytest.mark.parametrize("cols", [96, 70])
def test_a_nan_block_is_not_read_without_an_activation(B, cols):
    """x_act "none": dx is dy w, whatever was kept; dw is NaN in the lost columns alone."""
    x = matrix(40, cols, torch.bfloat16, 8)
    x[3, 40] = float("inf")
    q, w = B.checkpoint(x), matrix(24, cols, torch.bfloat16, 10)
    for rows in (40, 4):
        part, dy = B.Checkpoint(q.codes, q.scales, rows, cols), matrix(40, 24, torch.bfloat16, 11)[:rows]
        dx, dw, _ = B.linear_backward(dy, part, w)
        assert not torch.isnan(dx).any() and torch.equal(dx, B.linear(dy, w.t()))
        lost = torch.zeros(24, cols, dtype=torch.bool, device=DEV)
        lost[:, 32:64] = True
        assert torch.equal(torch.isnan(dw), lost)
