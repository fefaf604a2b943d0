"""MXFP4 quantisation, reading back and products against a plain implementation in 64 bits (numpy), written from the format: blocks
of 32, the smallest power-of-two scale (from 2^-127 on) for which six times it covers the block, elements on the grid
0, .5, 1, 1.5, 2, 3, 4, 6.

Quantised values have no tolerance.  Products: both operands are exact in fp32 and so is each product of two elements; what is
rounded is the sum of K products.  An fp32 sum of K terms in any order is off by at most (K - 1) 2^-24 of the sum of magnitudes
(first order); the tensor core may truncate instead of rounding: 2^-23 a step.  bf16 results add half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def philox(seed, c0, c1, c2, c3):
    """Philox4x32-10 on uint64 arrays of 32-bit words."""
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    m = np.uint64(0xFFFFFFFF)
    c0, c1, c2, c3 = (np.asarray(c, np.uint64) for c in (c0, c1, c2, c3))
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c0, np.uint64(0xCD9E8D57) * c2
        c0, c1, c2, c3 = (p1 >> np.uint64(32)) ^ c1 ^ np.uint64(k0), p1 & m, (p0 >> np.uint64(32)) ^ c3 ^ np.uint64(k1), p0 & m
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def bits16(rows, cols, seed, tag):
    g, r = np.meshgrid(np.arange(-(-cols // 8)), np.arange(rows))
    w = philox(seed, g, np.full_like(g, tag << 24), r, np.zeros_like(g))
    u = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], -1)
    return u.reshape(rows, -1)[:, :cols].astype(np.float64)


def quantise(x, u=None):
    """[rows, cols] in 64 bits -> (values, scale exponents [rows, blocks]); non-finite blocks are NaN (exponent 128)."""
    rows, cols = x.shape
    b = np.pad(x, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)
    nan = ~np.isfinite(b).all(-1)
    b = np.where(nan[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    k = np.full(top.shape, -127.0)
    live = top > 0
    k[live] = np.ceil(np.log2(top[live] / 6.0))
    k = np.where(live & (6.0 * np.exp2(k) < top), k + 1, k)
    k = np.where(live & (6.0 * np.exp2(k - 1) >= top), k - 1, k)
    k = np.maximum(k, -127.0)
    a = np.abs(b) / np.exp2(k)[..., None]
    lo = np.searchsorted(GRID, a, side="right") - 1
    hi = np.minimum(lo + 1, 7)
    gap = np.where(hi > lo, GRID[hi] - GRID[lo], 1.0)
    part = (a - GRID[lo]) / gap
    if u is None:
        up = (part > 0.5) | ((part == 0.5) & (lo % 2 == 1))
    else:
        up = part + np.pad(u, ((0, 0), (0, -cols % 32))).reshape(b.shape) / 65536 >= 1
    q = np.copysign(np.where(up, GRID[hi], GRID[lo]), b) * np.exp2(k)[..., None]
    q = np.where(nan[..., None], np.nan, q)
    return q.reshape(rows, -1)[:, :cols], np.where(nan, 128.0, k)


def untile(scales, rows, cols):
    blocks, kb = -(-cols // 32), -(-cols // 128)
    r, b = np.meshgrid(np.arange(rows), np.arange(blocks), indexing="ij")
    return scales[((r // 128) * kb + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4]


def decode(q):
    """Values and exponents of an MxTensor, from its bytes."""
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    pitch = 64 * -(-q.cols // 128)
    c = codes[: q.rows * pitch].reshape(q.rows, pitch)
    c = np.stack([c & 15, c >> 4], -1).reshape(q.rows, -1)
    assert not (c[:, q.cols:] & 7).any(), "the tail of a row must be zero"
    c = c[:, : q.cols].astype(np.int64)
    k = (untile(scales, q.rows, q.cols) if q.layout == "tiles" else scales.reshape(q.rows, -1)).astype(np.float64) - 127
    s = np.where(k == 128, np.nan, np.exp2(np.minimum(k, 127)))
    return np.where(c >> 3, -1.0, 1.0) * GRID[c & 7] * np.repeat(s, 32, 1)[:, : q.cols], k


def make(rows, cols, dtype, seed, extremes=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64) * torch.exp(2 * torch.randn(rows, 1, generator=g, dtype=torch.float64))
    x = x.to(dtype)
    if extremes and rows * cols > 400:
        f = x.view(-1)
        big, small = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
        f[5], f[69], f[133], f[197] = big, -big, small, 0.75 * small if dtype != torch.float16 else small
        f[256:290] = 0.0
        for i, v in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0)):     # every tie, with a top of six
            f[320 + i] = v
    return x


SIZES = [(1, 1), (1, 31), (1, 33), (1, 100003), (3, 128), (5, 129), (127, 32), (128, 128), (129, 257), (200, 4), (33, 1000), (700, 64), (1, 128), (128, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("layout", ["tiles", "linear"])
def test_quantised_values_are_exact(B, dtype, rows, cols, rounding, layout):
    x = make(rows, cols, dtype, rows + cols)
    seed = (1 << 40) + 12345
    xd = x.cuda()
    q, qt = B.mx_quantize(xd, along="both", rounding=rounding, seed=seed, layout=layout)
    alone, alone_t = (B.mx_quantize(xd, along=a, rounding=rounding, seed=seed, layout=layout) for a in ("rows", "cols"))
    x64 = x.double().numpy()
    for got, ref, tag in ((q, x64, 3), (alone, x64, 3), (qt, x64.T, 4), (alone_t, x64.T, 4)):
        u = bits16(*ref.shape, seed, tag) if rounding == "stochastic" else None
        want, k = quantise(ref, u)
        val, gk = decode(got)
        assert np.array_equal(gk, k)
        assert np.array_equal(val, want)
        for dt in (torch.float32, torch.bfloat16, torch.float16):
            back = B.mx_dequantize(got, dt).cpu()
            expect = torch.from_numpy(want).to(torch.float32).to(dt)             # fp32 holds the values exactly, or as a subnormal
            assert torch.equal(back, expect), dt


def test_strided_rows_and_untouched_neighbours(B):
    big = make(60, 200, torch.bfloat16, 3).cuda()
    for view in (big[:, 8:136], big[:, 3:100], big[::2, 40:41], big[7:8, 1:]):
        q, qt = B.mx_quantize(view, along="both")
        ref = view.double().cpu().numpy()
        assert np.array_equal(decode(q)[0], quantise(ref)[0]) and np.array_equal(decode(qt)[0], quantise(ref.T)[0])
        out = torch.full((view.shape[0], view.shape[1] + 5), 9.0, device="cuda")
        B.mx_dequantize(q, out=out[:, 2: 2 + view.shape[1]])
        # in the type of `out`: the largest bf16 is rounded to 4 * 2^126 in MXFP4, which fp32 reads as infinity
        with np.errstate(over="ignore"):
            assert np.array_equal(out[:, 2: 2 + view.shape[1]].cpu().numpy(), quantise(ref)[0].astype(np.float32))
        assert (out[:, :2] == 9).all() and (out[:, 2 + view.shape[1]:] == 9).all()
    with pytest.raises(ValueError):
        B.mx_quantize(big.t())


def test_non_finite_blocks_read_as_nan(B):
    x = torch.ones(3, 96)
    x[0, 40], x[1, 0], x[2, 95] = float("inf"), float("nan"), float("-inf")
    q, qt = B.mx_quantize(x.cuda(), along="both")
    for t, ref in ((q, x.double().numpy()), (qt, x.double().numpy().T)):
        want = quantise(ref)[0]
        assert np.isnan(want).any() and np.array_equal(decode(t)[0], want, equal_nan=True)
        assert np.array_equal(B.mx_dequantize(t).double().cpu().numpy(), want, equal_nan=True)


def test_stochastic_rounding_is_unbiased(B):
    """1.3 of a block whose top is 6 (scale 1) goes to 1.5 with probability 0.6: mean over 2^20 draws within five deviations
    (0.5 sqrt(0.24) / 2^10 = 0.00024)."""
    x = torch.full((1 << 15, 32), 1.3)
    x[:, 0] = 6.0
    back = B.mx_dequantize(B.mx_quantize(x.cuda(), rounding="stochastic", seed=5))[:, 1:].double()
    assert abs(back.mean().item() - 1.3) < 0.0012
    other = B.mx_dequantize(B.mx_quantize(x.cuda(), rounding="stochastic", seed=6))[:, 1:].double()
    assert not torch.equal(back, other)


def product_case(B, M, N, K, dtype, seed=0, out=None):
    g = torch.Generator().manual_seed(seed + 7 * M + N + K)
    a = torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, 1, generator=g))
    b = torch.randn(N, K, generator=g) * torch.exp(torch.randn(N, 1, generator=g))
    qa, qb = B.mx_quantize(a.cuda()), B.mx_quantize(b.cuda())
    got = B.mx_matmul(qa, qb, dtype, out=out)
    va, vb = quantise(a.double().numpy())[0], quantise(b.double().numpy())[0]
    want, size = va @ vb.T, np.abs(va) @ np.abs(vb).T
    off = np.abs(got.double().cpu().numpy() - want)
    tol = K * 2.0 ** -23 * size + (2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -7) if got.dtype == torch.bfloat16 else 0)
    bad = off > tol
    assert not bad.any(), (M, N, K, int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(off.max()), float((off / np.maximum(size, 1e-30)).max()))
    return got


# all widths of B's tile (16, 32, 64, 128, 256), both roles, ragged and tiny sizes, k of one block to many, split and whole
PRODUCTS = [(1, 1, 1), (1, 128, 32), (1, 1000, 4096), (2, 300, 500), (16, 256, 256), (17, 129, 1000), (31, 500, 130), (33, 1000, 700), (64, 640, 2048),
            (65, 100, 300), (100, 65, 260), (128, 128, 128), (129, 257, 385), (300, 7, 900), (500, 40, 1500), (1000, 64, 64), (257, 129, 33),
            (1500, 3000, 128), (2050, 2047, 515), (2500, 2600, 200), (2561, 5130, 140), (5000, 1, 200), (1, 20000, 160)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_products_match(B, M, N, K, dtype):
    product_case(B, M, N, K, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(2050, 2047, 4200), (2300, 2305, 515), (1281, 2049, 8000)])
def test_products_of_a_few_large_tiles(B, M, N, K, dtype):
    """One or two rounds of the large tiles, ragged on every side: chosen for long sums, or once the small tiles need a second wave."""
    product_case(B, M, N, K, dtype)


@pytest.mark.parametrize("M,N,K", [(4096, 8192, 2048), (8192, 8192, 512), (2816, 5376, 4100)])
def test_many_tiles_a_multiprocessor(B, M, N, K):
    """Several rounds of tiles for every pair of multiprocessors, so that each role of the kernel runs into the next tile, with
    block scales spread over 2^6 so that a scale of another block shows.  Reference in fp32 on the values read back (its own sums
    are off by as much as the kernel's may be: twice the tolerance), four runs."""
    g = torch.Generator(device="cuda").manual_seed(M + K)

    def operand(rows):
        spread = torch.exp2(torch.randint(-3, 4, (rows, -(-K // 32), 1), generator=g, device="cuda").float()).expand(-1, -1, 32).reshape(rows, -1)[:, :K]
        return B.mx_quantize(torch.randn(rows, K, generator=g, device="cuda") * spread)

    a, b = operand(M), operand(N)
    va, vb = B.mx_dequantize(a), B.mx_dequantize(b)
    want, tol = va @ vb.t(), 2 * K * 2.0 ** -23 * (va.abs() @ vb.abs().t())
    for _ in range(4):
        outs = [B.mx_matmul(a, b, torch.float32) for _ in range(3)]
        assert all(bool(((o - want).abs() <= tol).all()) for o in outs)


def test_product_into_strided_rows_leaves_the_rest(B):
    for M, N in ((3, 200), (130, 190), (200, 33)):
        out = torch.full((M, N + 11), 5.0, device="cuda")
        product_case(B, M, N, 600, None, out=out[:, 4: 4 + N])
        assert (out[:, :4] == 5).all() and (out[:, 4 + N:] == 5).all()


def test_products_are_the_same_bits_each_time_and_from_a_graph(B):
    x, w = torch.randn(9, 3000, device="cuda"), torch.randn(700, 3000, device="cuda")
    qw = B.mx_quantize(w)
    first = B.mx_matmul(B.mx_quantize(x), qw, torch.float32).clone()
    for _ in range(3):
        assert torch.equal(first, B.mx_matmul(B.mx_quantize(x), qw, torch.float32))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = B.mx_matmul(B.mx_quantize(x), qw, torch.float32)
    x.mul_(2.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, 2 * first)             # a power of two moves the scales only
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z = B.mx_matmul(B.mx_quantize(x, stream=side), qw, torch.float32, stream=side)
    side.synchronize()
    assert torch.equal(z, y)


def test_products_on_two_streams_at_once(B):
    """A large product (pairs of multiprocessors, all of their tensor memory), small ones and quantisations, interleaved on two
    streams: nothing is shared, and each result is what it is alone."""
    big = [B.mx_quantize(torch.randn(n, 1500, device="cuda")) for n in (2500, 2600)]
    small = [B.mx_quantize(torch.randn(n, 3000, device="cuda")) for n in (20, 700)]
    x = torch.randn(300, 1100, device="cuda")
    calls = (lambda st: B.mx_matmul(*big, torch.float32, stream=st), lambda st: B.mx_matmul(*small, torch.float32, stream=st),
             lambda st: B.mx_dequantize(B.mx_quantize(x, along="cols", stream=st), stream=st))
    alone = [c(None).clone() for c in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for i in range(12):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[k].append(((i + k) % 3, calls[(i + k) % 3](None)))
    torch.cuda.synchronize()
    assert all(torch.equal(out, alone[c]) for part in got for c, out in part)


def test_zero_and_nan_rows_in_a_product(B):
    a, b = torch.randn(40, 160), torch.randn(70, 160)
    a[3], b[5] = 0.0, 0.0
    a[7, 100], b[9, 31] = float("nan"), float("inf")
    y = B.mx_matmul(B.mx_quantize(a.cuda()), B.mx_quantize(b.cuda()), torch.float32).cpu()
    assert torch.isnan(y[7]).all() and torch.isnan(y[:, 9]).all()
    rest = [i for i in range(40) if i != 7]
    cols = [j for j in range(70) if j != 9]
    assert torch.isfinite(y[rest][:, cols]).all()
    assert not y[3, cols].any() and not y[rest, 5].any()


def test_a_layer_trained_in_four_bits(B):
    """Output and both gradients of y = x w^T from three quantisations, as a training step calls them; the gradients against the
    formula's on the quantised operands and against a difference of the quantised loss in the direction of dy."""
    M, N, K = 150, 90, 70
    g = torch.Generator().manual_seed(1)
    x, w, dy = torch.randn(M, K, generator=g), torch.randn(N, K, generator=g), torch.randn(M, N, generator=g)
    (x4, x4t), (w4, w4t) = (B.mx_quantize(t.cuda(), along="both") for t in (x, w))
    dy4, dy4t = B.mx_quantize(dy.cuda(), along="both", rounding="stochastic", seed=3)
    y, dx, dw = B.mx_matmul(x4, w4, torch.float32), B.mx_matmul(dy4, w4t, torch.float32), B.mx_matmul(dy4t, x4t, torch.float32)
    n = {k: t.double().numpy() for k, t in (("x", x), ("w", w), ("dy", dy))}
    q = lambda t, u=None: quantise(t, u)[0]  # noqa: E731
    for got, a, b in ((y, q(n["x"]), q(n["w"])), (dx, q(n["dy"], bits16(M, N, 3, 3)), q(n["w"].T)), (dw, q(n["dy"].T, bits16(N, M, 3, 4)), q(n["x"].T))):
        size = np.abs(a) @ np.abs(b).T
        assert np.all(np.abs(got.double().cpu().numpy() - a @ b.T) <= a.shape[1] * 2.0 ** -23 * size)
    # loss(x) = sum(dy4 * (x w4t^T)) is linear in x: its difference along any direction is that direction with dx
    d = np.random.default_rng(0).standard_normal((M, K))
    dyv, wv = q(n["dy"], bits16(M, N, 3, 3)), q(n["w"].T).T
    loss = lambda t: float((dyv * (t @ wv.T)).sum())  # noqa: E731
    diff = (loss(n["x"] + 1e-3 * d) - loss(n["x"] - 1e-3 * d)) / 2e-3
    slack = N * 2.0 ** -23 * float((np.abs(d) * (np.abs(dyv) @ np.abs(wv))).sum()) + 1e-9 * abs(diff)
    assert abs(diff - float((dx.double().cpu().numpy() * d).sum())) <= slack


def test_a_pushed_gradient_reaches_the_parameters(B):
    """A worker's weight gradient, pushed in 4 bits, averaged with another worker's and stepped with AdamW: as used together."""
    n = 50 * 70
    grads = [torch.randn(50, 70, device="cuda") for _ in range(2)]
    pushes = [[B.mx_quantize(g.view(-1), layout="linear", rounding="stochastic", seed=i)] for i, g in enumerate(grads)]
    p = torch.zeros(n, device="cuda")
    opt = B.AdamW([p], pushes, weight_decay=0.0)
    opt.step(1, 0.1)
    mean = sum(B.mx_dequantize(q[0]).view(-1) for q in pushes) / 2
    want = -0.1 * mean / (mean.abs() + 1e-8)
    assert torch.all((p - want).abs() <= 0.1 * 2.0 ** -18)


def test_results_on_a_given_stream_are_its_own(B):
    """A buffer freed while its stream still writes it must not become the result of a call on another stream, and an operand dropped
    after its call must not be overwritten before that stream has read it."""
    x = torch.randn(1024, 4096, device="cuda")
    want = B.mx_quantize(x)
    back, prod = B.mx_dequantize(want), B.mx_matmul(want, want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def busy(shape, dtype):               # memory that the current stream fills some milliseconds later, handed back at once
        t = torch.empty(shape, dtype=dtype, device="cuda")
        torch.cuda._sleep(20_000_000)
        t.fill_(7)

    for t in (want._buffer, back, prod):
        busy(1, t.dtype)                  # a kernel's first launch waits for the device
    torch.cuda.synchronize()
    busy(want._buffer.shape, torch.uint8)
    q = B.mx_quantize(x, stream=side)
    busy(back.shape, back.dtype)
    r = B.mx_dequantize(want, stream=side)
    busy(prod.shape, prod.dtype)
    c = B.mx_matmul(want, want, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(q._buffer, want._buffer) and torch.equal(r, back) and torch.equal(c, prod)
    y, q2 = x.clone(), B.mx_quantize(x)
    torch.empty_like(x).zero_()
    torch.empty_like(want._buffer).zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    q = B.mx_quantize(y, stream=side)
    r = B.mx_dequantize(q2, stream=side)
    del y, q2
    torch.empty_like(x).zero_()
    torch.empty_like(want._buffer).zero_()
    torch.cuda.synchronize()
    assert torch.equal(q._buffer, want._buffer) and torch.equal(r, back)


def test_refusals(B):
    x = torch.randn(4, 64, device="cuda")
    q = B.mx_quantize(x)
    for bad in (lambda: B.mx_quantize(x.double()), lambda: B.mx_quantize(x.cpu()), lambda: B.mx_quantize(x[:0]), lambda: B.mx_quantize(x.view(2, 2, 64)),
                lambda: B.mx_quantize(x, along="all"), lambda: B.mx_quantize(x, rounding="down"), lambda: B.mx_quantize(x, layout="rows"),
                lambda: B.mx_matmul(q, B.mx_quantize(x[:, :32])), lambda: B.mx_matmul(q, B.mx_quantize(x, layout="linear")), lambda: B.mx_matmul(q, q, torch.float16),
                lambda: B.mx_matmul(q, q, out=torch.empty(4, 5, device="cuda")), lambda: B.mx_dequantize(q, torch.float64), lambda: B.mx_dequantize(q, out=x.t()),
                lambda: B.MxTensor(q.codes, q.scales, 4, 200, "tiles"), lambda: B.MxTensor(q.codes, q.scales, 129, 64, "tiles"), lambda: B.MxTensor(q.codes, q.scales, 4, 64, "x")):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("M,N,K", [(1500, 1600, 1 << 23), (1, 128, 1 << 26)])
def test_very_long_sums(B, M, N, K):
    """Tiles that take tens of milliseconds: the bounded waits for them do not run out.  Ones only: every partial sum is exact."""
    def ones(rows):
        codes = torch.full((rows * K // 2,), 0x22, dtype=torch.uint8, device="cuda")
        scales = torch.full((-(-rows // 128) * (K // 128) * 512,), 127, dtype=torch.uint8, device="cuda")
        return B.MxTensor(codes, scales, rows, K, "tiles")
    c = B.mx_matmul(ones(M), ones(N), torch.float32)
    assert torch.all(c == float(K))
    torch.cuda.empty_cache()


def test_offsets_beyond_32_bits(B):
    """A flat vector and a matrix of more than 2^32 bytes and elements: their ends are those of a small call on the same values."""
    n = (1 << 31) + 77
    x = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = 64 * 40 + 77 - 64
    x[-tail:] = torch.randn(tail, device="cuda").bfloat16()
    q = B.mx_quantize(x, layout="linear")
    small = B.mx_quantize(x[n - tail:].clone(), layout="linear")
    assert (n - tail) % 32 == 0
    got, want = B.mx_dequantize(q, torch.bfloat16)[0, n - tail:], B.mx_dequantize(small, torch.bfloat16)[0]
    assert torch.equal(got, want) and want.any()
    del x, q, got
    torch.cuda.empty_cache()
    rows, cols = 66000, 65600                    # 4.3e9 elements
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-40:] = torch.randn(40, cols, device="cuda").bfloat16()
    q, qt = B.mx_quantize(x, along="both")
    back = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    B.mx_dequantize(q, out=back)
    small = B.mx_dequantize(B.mx_quantize(x[-40:].clone()), torch.bfloat16)
    assert torch.equal(back[-40:], small) and not back[-41].any()
    # the transpose's last row: column cols - 1, whose only entries are the last 40 (blocks of 32 rows: 65984.., 65952..)
    y = B.mx_matmul(q, B.mx_quantize(torch.ones(1, cols, device="cuda")), torch.float32)
    want = small.double().sum(1)
    size = small.double().abs().sum(1)
    assert torch.all((y[-40:, 0].double() - want).abs() <= cols * 2.0 ** -23 * size) and not y[:-40].any()
    del back
    t = B.mx_dequantize(qt, torch.bfloat16)
    ref = quantise(x[65952:, -1:].double().cpu().numpy().T)[0]
    assert np.array_equal(t[-1, 65952:].double().cpu().numpy(), ref[0])
    del x, q, qt, t, y
    torch.cuda.empty_cache()
