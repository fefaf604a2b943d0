"""Ends of the worker's operators' ranges: the smallest sizes, the shapes at which the products change their way, residuals in place in every type, calls side by side.

Tolerances as in the products' tests."""
import numpy as np
import pytest
import torch

from test_gpu_worker_linear import check_linear, normal, sum_tol
from worker_ref import EPS, TINY, act, close, f64, keep, slope, values

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (2, 1, 3), (1, 3, 1), (17, 2, 1), (65, 64, 1), (129, 1, 129), (300, 1, 2), (128, 64, 32), (128, 64, 33), (128, 65, 64), (64, 63, 64), (64, 64, 63)])
def test_smallest_sizes(B, M, K, N):
    gen = torch.Generator(device=DEV).manual_seed(M + 3 * K + 5 * N)
    x, w = normal(gen, M, K), normal(gen, N, K)
    check_linear(B, x, w, normal(gen, N, dtype=torch.float32), "silu", normal(gen, M, N), keep_z=True)
    dy = normal(gen, M, N)
    dx, dw, db = B.linear_backward(dy, B.checkpoint(x), w, x_act="gelu")
    V, G, W = keep(f64(x))[0], f64(dy), f64(w)
    want, s = (G @ W) * slope("gelu", V), np.abs(slope("gelu", V))
    close(dx, want, sum_tol(G, W.T) * (s + 2.0**-14) * 1.01 + np.abs(G @ W) * 2.0**-14 + 2.0**-8 * np.abs(want) + TINY[torch.bfloat16], "dx")
    H = f64(B.checkpoint_read(B.checkpoint(x), torch.bfloat16, act="gelu"))
    close(dw, G.T @ H, sum_tol(G.T, H.T) * 1.01 + 2.0**-24 * np.abs(G.T @ H), "dw")
    close(db, G.sum(0), M * 2.0**-24 * np.abs(G).sum(0) * 1.01, "db")


# one more or less than: few rows / tiles, one cluster / several, tiles / pairs, one and two blocks a multiprocessor
@pytest.mark.parametrize("M,K,N", [(64, 4096, 640), (65, 4096, 640), (16, 8192, 200), (32, 8192, 200), (33, 520, 19000), (1, 264, 50000), (1, 72, 20000), (1792, 192, 1792), (1793, 192, 2049), (600, 3200, 600), (256, 6400, 128), (2049, 128, 1793)])
@pytest.mark.parametrize("odt", ["same", "f32"])
def test_where_the_way_changes(B, M, K, N, odt):
    gen = torch.Generator(device=DEV).manual_seed(M + K + N)
    dt = torch.bfloat16 if N % 2 else torch.float16
    odt = dt if odt == "same" else torch.float32
    x, w, r = normal(gen, M, K, dtype=dt), normal(gen, N, K, dtype=dt, scale=K**-0.5), normal(gen, M, N, dtype=odt)
    want = check_linear(B, x, w, normal(gen, N, dtype=dt), "relu", r, keep_z=True, dtype=odt)
    plain = B.linear(x, w, residual=r, dtype=odt)
    c = r.clone()
    assert torch.equal(B.linear(x, w, residual=c, out=c), plain) and want.dtype == odt


def test_calls_side_by_side(B):
    """The same calls on four streams at once, each with results of its own: the bits of the calls one by one."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    jobs = [(normal(gen, M, K), normal(gen, N, K, scale=0.1)) for M, K, N in ((3, 4097, 900), (300, 3000, 700), (1500, 600, 2100), (64, 512, 64))]
    logits = normal(gen, 40, 20001)
    tokens = torch.arange(40, device=DEV)

    def all_of(x, w):
        y, z = B.linear(x, w, act="gelu", keep=True)
        g = B.linear_backward(y, B.checkpoint(x), w, x_act="silu")
        p = B.log_probs(logits, tokens, top=5, d_logp=torch.ones(40, device=DEV))
        return [y, z.codes, z.scales, *g, p.logp, p.top_ids, p.dlogits]

    want = [all_of(x, w) for x, w in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for st, (x, w) in zip(streams, jobs):
            with torch.cuda.stream(st):
                got.append(all_of(x, w))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_kept_values_in_place_of_the_tensor(B):
    """A Checkpoint made from the caller's own bytes, longer than needed, reads as the one it came from."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    x = normal(gen, 37, 100)
    q = B.checkpoint(x)
    codes, scales = torch.zeros(q.codes.numel() + 64, dtype=torch.uint8, device=DEV), torch.zeros(q.scales.numel() + 5, dtype=torch.uint8, device=DEV)
    codes[: q.codes.numel()], scales[: q.scales.numel()] = q.codes, q.scales
    mine = B.Checkpoint(codes, scales, 37, 100)
    assert torch.equal(mine.codes, q.codes) and torch.equal(mine.scales, q.scales)
    assert torch.equal(B.checkpoint_read(mine, act="gelu"), B.checkpoint_read(q, act="gelu")) and np.array_equal(values(mine)[0], keep(f64(x))[0])
    with pytest.raises(ValueError):
        B.Checkpoint(codes[:100], scales, 37, 100)
    with pytest.raises(B.SimError):                # off 16-byte boundaries
        B.checkpoint_read(B.Checkpoint(codes[8: 8 + q.codes.numel()], scales, 37, 100))


def test_refusals_on_the_device(B):
    gen = torch.Generator(device=DEV).manual_seed(6)
    x, w = normal(gen, 4, 32), normal(gen, 8, 32)
    q = B.checkpoint(x)
    for call in (lambda: B.linear(x, w.half()), lambda: B.linear(x, w[:, :16]), lambda: B.linear(x.float(), w.float()), lambda: B.linear(x, w, dtype=torch.float16), lambda: B.linear(x, w, residual=normal(gen, 4, 7)),
                 lambda: B.linear(x, w, residual=normal(gen, 4, 8, dtype=torch.float32)), lambda: B.linear(x, w, normal(gen, 9)), lambda: B.linear(x, w, normal(gen, 8, dtype=torch.float16)),
                 lambda: B.linear(x, w, out=torch.zeros(4, 9, device=DEV)), lambda: B.linear(x.expand(2, 4, 32), w), lambda: B.linear(x[:1].expand(4, 32), w), lambda: B.linear(x, w, act="swish"),
                 lambda: B.linear(x, w.cpu()), lambda: B.linear_backward(normal(gen, 4, 8), x, w, x_act="gelu"), lambda: B.linear_backward(normal(gen, 4, 9), x, w), lambda: B.linear_backward(normal(gen, 4, 8), q, w, need="q"),
                 lambda: B.linear_backward(normal(gen, 8, 4).t(), q, w), lambda: B.act_backward(x, B.checkpoint(w), "relu"), lambda: B.log_probs(x, torch.zeros(3, dtype=torch.int64, device=DEV)),
                 lambda: B.log_probs(x, top=33), lambda: B.log_probs(x, d_logp=torch.zeros(4, device=DEV)), lambda: B.log_probs(x, out=x), lambda: B.log_probs(x, torch.zeros(4, device=DEV)),
                 lambda: B.log_probs_backward(x, None), lambda: B.checkpoint_read(q, torch.int8)):
        with pytest.raises(ValueError):
            call()
    buf = normal(gen, 4, 64)
    for call in (lambda: B.linear(buf[:, :32], w, out=buf[:, 16:24]), lambda: B.log_probs(buf[:, :32], torch.zeros(4, dtype=torch.int64, device=DEV), d_logp=torch.zeros(4, device=DEV), out=buf[:, 1:33]),
                 lambda: B.log_probs(x, temperature=0.0), lambda: B.checkpoint_read(q, out=q.codes.view(torch.bfloat16)[:64].view(2, 32).repeat(2, 1)[:3])):
        with pytest.raises((B.SimError, ValueError)):
            call()


def test_results_in_buffers_that_are_read_or_shared(B):
    """Column slices of one buffer hold operand and result; a gradient over the input that another gradient still needs is refused, over one that nothing needs it is not."""
    gen = torch.Generator(device=DEV).manual_seed(7)
    T, n = 70, 64
    x, w, dy = normal(gen, T, n), normal(gen, n, n), normal(gen, T, n)
    want = B.linear_backward(dy, x, w)
    buf = torch.zeros(T, 4 * n, dtype=torch.bfloat16, device=DEV)
    buf[:, n: 2 * n] = x
    B.linear(buf[:, n: 2 * n], w, act="gelu", out=buf[:, 2 * n: 3 * n])
    dx, dw, db = B.linear_backward(dy, buf[:, n: 2 * n], w, out=(buf[:, :n], None, None))
    assert torch.equal(buf[:, 2 * n: 3 * n], B.linear(x, w, act="gelu")) and torch.equal(buf[:, n: 2 * n], x) and not buf[:, 3 * n:].any()
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), want))
    one = torch.empty(T, n, dtype=torch.bfloat16, device=DEV)
    for out in ((x, None, None), (x[:, :], None, None), (None, None, w[0]), (None, None, dy[0]), (one, one[:n], None), (one, None, one[0]), (None, one[:n], one[1])):
        with pytest.raises((ValueError, B.SimError)):
            B.linear_backward(dy, x, w, out=out, dtype=torch.bfloat16)
    assert torch.equal(buf[:, n: 2 * n], x)
    got = B.linear_backward(dy, x, w, need="x", out=(x, None, None))[0]
    assert got is x and torch.equal(x, want[0])


def test_copied_operands_replayed(B):
    """Operands off 16-byte boundaries, whose copies the products overtake: captured once, replayed behind one another over changing inputs."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    for T, fin, fout in ((37, 333, 1003), (1800, 521, 2049)):
        x, w, dy = normal(gen, T, fin), normal(gen, fout, fin, scale=0.05), normal(gen, T, fout)
        B.linear_backward(dy, x, w)                  # loads the kernels
        B.linear(x, w)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = B.linear(x, w, act="silu")
            got = (y,) + B.linear_backward(dy, x, w)
        runs = [(normal(gen, T, fin), normal(gen, fout, fin, scale=0.05), normal(gen, T, fout)) for _ in range(4)]
        want = [(B.linear(a, b, act="silu"),) + B.linear_backward(c, a, b) for a, b, c in runs]
        out = []
        for a, b, c in runs:
            x.copy_(a), w.copy_(b), dy.copy_(c)
            g.replay()
            out.append([t.clone() for t in got])
        torch.cuda.synchronize()
        for o, e in zip(out, want):
            assert all(torch.equal(u, v) for u, v in zip(o, e))
