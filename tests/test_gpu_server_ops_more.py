"""More of the server's operators: unaligned lists of every push type, lists that mix all types, betas of zero, the documented rounding of 8-bit
states bit for bit, its bias, and large products between guard elements.  References in 64 bits; tolerances in each test."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import Case, F32, decode8, e4m3, mx_decode, reference
from test_gpu_mx import philox, product_case

pytestmark = pytest.mark.gpu
CODES = e4m3(np.arange(127))                       # the non-negative E4M3 values, 0 to 448


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("g_type", [torch.float32, torch.bfloat16, torch.float16, "mx"])
@pytest.mark.parametrize("K", [1, 3])
def test_unaligned_lists_of_every_push_type(B, bits, p_type, g_type, K):
    """Tensors one element apart (pushes in MXFP4: at any byte), with the bf16 copy: values, and everything between the tensors untouched."""
    c = Case(B, [1, 7, 33, 2049, 300, 5, 4100], p_type, g_type, K, bits, gap=1, seed=11 + K, shadow=p_type == torch.float32)
    marks = torch.ones(c.flat_p.numel(), dtype=torch.bool)
    for o, n in zip(c.offs, c.sizes):
        marks[o: o + n] = False
    flats = [c.flat_p, c.flat["m"], c.flat["v"]] + ([c.flat_shadow] if c.flat_shadow is not None else [])
    old = [t.clone() for t in flats]
    for t in (1, 500):
        before = c.snapshot()
        c.opt.step(t, 3e-3, grad_scale=0.5)
        torch.cuda.synchronize()
        c.check(before, float(np.float32(3e-3)), t, 0.5)
    for a, b in zip(old, flats):
        assert torch.equal(a.cpu()[marks], b.cpu()[marks]) and not torch.equal(a, b)
    c.opt.close()


def mixed(B, bits, K, betas=(0.9, 0.999), decay=0.1):
    """One tensor of each pair of types, aligned and not, of several lengths, in one list."""
    rng = np.random.default_rng(bits + K)
    ps, pushes, shadow = [], [[] for _ in range(K)], []
    combos = [(p, g, at) for at in (0, 1) for p in (torch.float32, torch.bfloat16) for g in (torch.float32, torch.bfloat16, torch.float16, "mx")]
    for i, (p_type, g_type, at) in enumerate(combos):
        n = (2048, 1, 3000, 33)[i % 4] + i
        flat = lambda dt, s: torch.from_numpy(rng.standard_normal(n + 8) * s).cuda().to(dt)[at: at + n]  # noqa: E731
        ps.append(flat(p_type, 0.1))
        for l in range(K):
            if g_type == "mx":
                pushes[l].append(B.mx_quantize(torch.from_numpy(rng.standard_normal(n) * 1e-2).cuda().float(), layout="linear"))
            else:
                pushes[l].append(flat(g_type, 1e-2))
        shadow.append(torch.zeros(n, dtype=torch.bfloat16, device="cuda") if p_type == torch.float32 else None)
    opt = B.AdamW(ps, pushes, betas=betas, weight_decay=decay, state_bits=bits, shadow=shadow, seed=5)
    grads = [[mx_decode(g.codes.cpu().numpy(), g.scales.cpu().numpy(), p.numel()) if isinstance(g, B.MxTensor) else g.double().cpu().numpy() for g in (push[i] for push in pushes)]
             for i, p in enumerate(ps)]
    return opt, grads


def moments(opt, i):
    s = {k: opt.state[k][i].cpu().numpy() for k in opt.state}
    if opt.state_bits == 32:
        return s["m"].astype(np.float64), s["v"].astype(np.float64)
    return decode8(s["m"], s["m_scale"]), decode8(s["v"], s["v_scale"]) ** 2


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("K", [1, 3])
@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.0, 0.0), (0.0, 0.99), (0.9, 0.0)])
def test_a_list_of_all_types_at_once(B, bits, K, betas):
    """Each tensor of a list that takes a launch per pair of types, betas of zero among them.  Roundings as in test_gpu_adamw: 2^-20 of the largest
    magnitude involved, where pushes cancel the fraction c2 |g| gm / v more (derived there), and half a step for bf16 parameters."""
    opt, grads = mixed(B, bits, K, betas)
    b1, b2 = betas
    lr = float(np.float32(1e-2))
    for t in (1, 2, 30):
        before = [(p.double().cpu().numpy(), *moments(opt, i)) for i, p in enumerate(opt.params)]
        opt.step(t, 1e-2)
        torch.cuda.synchronize()
        for i, (p0, m0, v0) in enumerate(before):
            want, m, v = reference(p0, m0, v0, grads[i], lr, t, 0.1, b1, b2)
            got = opt.params[i].double().cpu().numpy()
            gm, g = sum(np.abs(x) for x in grads[i]) / K, np.abs(sum(grads[i]) / K)
            top = lr * (b1 * np.abs(m0) + (1 - b1) * gm) / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + 1e-8)
            top = np.abs(p0) + top * (1 + (1 - b2) * g * gm / np.maximum(v, 1e-300))
            tol = F32 * top + (2.0 ** -8 * np.abs(want) if opt.params[i].dtype == torch.bfloat16 else 0)
            assert np.all(np.abs(got - want) <= tol), (i, t, np.abs(got - want).max())
            if opt.shadow[i] is not None:
                assert torch.equal(opt.shadow[i], opt.params[i].to(torch.bfloat16))
            if bits == 32:
                gm_m, gm_v = moments(opt, i)
                assert np.all(np.abs(gm_m - m) <= F32 * (np.abs(m0) + gm + 1e-30)) and np.all(np.abs(gm_v - v) <= F32 * (v0 + gm * gm + 1e-30))
    opt.close()


def halves(n, seed, step, tensor):
    """The documented 16-bit numbers of a tensor's elements: counter (element / 8, tag 2, step, index in the list)."""
    g = np.arange(-(-n // 8), dtype=np.uint64)
    w = philox(seed, g, np.full_like(g, 2 << 24), np.full_like(g, step), np.full_like(g, tensor))
    return np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], -1).reshape(-1)[:n].astype(np.int64)


def encode8(x, u, keep):
    """Codes and scale bytes of x under stochastic rounding with u, and which elements and blocks are decided with a margin: of 2^-13 of a step from
    their threshold, and (keep: x is a root, off by 2^-22) of 2^-21 from a top of exactly 448 scales."""
    n = x.size
    top = np.abs(np.pad(x, (0, -n % 32))).reshape(-1, 32).max(1)
    k = np.full(top.shape, -127.0)
    live = top > 0
    k[live] = np.maximum(np.ceil(np.log2(top[live] / 448.0)), -127)
    sure_block = np.abs(top / (448 * np.exp2(k)) - 1) > 2.0 ** -21 if keep else np.ones(top.shape, bool)
    a = np.abs(x) / np.repeat(np.exp2(k), 32)[:n]
    lo = np.searchsorted(CODES, a, side="right") - 1
    hi = np.minimum(lo + 1, 126)
    part = (a - CODES[lo]) / np.where(hi > lo, CODES[hi] - CODES[lo], 1.0) + u / 65536
    code = np.where(part >= 1, hi, lo)
    if keep:
        code = np.where((code == 0) & (a > 0), 1, code)
    return code | np.where(np.signbit(x), 128, 0), (k + 127).astype(np.int64), (np.abs(part - 1) > 2.0 ** -13) & np.repeat(sure_block, 32)[:n], sure_block


@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("K", [1, 2])
def test_eight_bit_states_are_rounded_as_documented(B, at, K):
    """Codes and scale bytes bit for bit.  Pushes are whole multiples of 2^-10 and betas powers of two, so that m is exact in fp32 and r = sqrt(v) off by
    the root's 2^-22 alone, at most 2^-18 of a step: elements within 2^-13 of a step of their threshold are left out (about one in 4000), and for r blocks
    whose top is 448 scales to within that error (of multiples of 2^-10 several in a hundred are exactly that).  The second step
    starts from stored states (b2 = 0: its r is |g|).  at = 1: unaligned, the same numbers by element."""
    n, seed, lr = 9001, (1 << 45) + 77, 0.5
    rng = np.random.default_rng(8)
    g = [np.round(rng.standard_normal(n) * np.exp2(rng.integers(-4, 5, n))) * 8 + rng.integers(1, 8, n) for _ in range(K)]
    g = [(x * 2.0 ** -10).astype(np.float32) for x in g]
    place = lambda a, dt: torch.zeros(n + 40, dtype=dt, device="cuda")[at: at + n].copy_(torch.from_numpy(a))  # noqa: E731
    first = torch.zeros(40, device="cuda")
    p, pushes = place(np.zeros(n, np.float32), torch.float32), [place(x, torch.float32) for x in g]
    state = {"m": [torch.zeros(40, dtype=torch.uint8, device="cuda"), place(np.zeros(n, np.uint8), torch.uint8)],
             "v": [torch.zeros(40, dtype=torch.uint8, device="cuda"), place(np.zeros(n, np.uint8), torch.uint8)]}
    state |= {k: [torch.zeros(2, dtype=torch.uint8, device="cuda"), torch.zeros(-(-n // 32), dtype=torch.uint8, device="cuda")] for k in ("m_scale", "v_scale")}
    mean = sum(x.astype(np.float64) for x in g) / K
    m = np.zeros(n)
    for t, b2 in ((1, 0.75), (2, 0.0)):
        opt = B.AdamW([first, p], [[torch.zeros_like(first), x] for x in pushes], betas=(0.5, b2), weight_decay=0.0, state_bits=8, state=state, seed=seed)
        opt.step(t, lr)
        torch.cuda.synchronize()
        m, r = 0.5 * m + 0.5 * mean, np.sqrt(1 - b2) * np.abs(mean)
        u = halves(n, seed, t, 1)
        got = {k: v[1].cpu().numpy().astype(np.int64) for k, v in state.items()}
        for name, x, bits, keep in (("m", m, u, False), ("v", r, (u & 255) << 8 | u >> 8, True)):
            codes, scales, sure, blocks = encode8(x, bits, keep)
            assert np.array_equal(got[name + "_scale"][blocks], scales[blocks]), (name, t)
            sure &= x != 0                             # a zero's sign says nothing
            assert sure.mean() > 0.9 and np.array_equal(got[name][sure], codes[sure]), (name, t)
        m = decode8(state["m"][1].cpu().numpy(), state["m_scale"][1].cpu().numpy())
        opt.close()


@pytest.mark.parametrize("at", [0, 1])
def test_the_first_moment_decays_without_bias(B, at):
    """As the second moment in test_gpu_adamw (same bound): with zero gradients m follows 0.999^t on average, aligned or not."""
    n = 65536
    flat = lambda dt: torch.zeros(n + 8, dtype=dt, device="cuda")[at: at + n]  # noqa: E731
    p, g = flat(torch.float32), flat(torch.float32)
    state = {"m": [flat(torch.uint8)], "v": [flat(torch.uint8)]} | {k: [torch.zeros(n // 32, dtype=torch.uint8, device="cuda")] for k in ("m_scale", "v_scale")}
    opt = B.AdamW([p], [[g]], state_bits=8, state=state, betas=(0.999, 0.999), weight_decay=0.0, seed=12)
    g.fill_(-1.0)
    opt.step(1, 0.0)
    g.zero_()
    m0 = decode8(state["m"][0].cpu().numpy(), state["m_scale"][0].cpu().numpy()).mean()
    for t in range(2, 202):
        opt.step(t, 0.0)
    m = decode8(state["m"][0].cpu().numpy(), state["m_scale"][0].cpu().numpy()).mean()
    assert m0 < 0 and abs(m / m0 / 0.999 ** 200 - 1) < 0.01


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K,col", [(2500, 2600, 200, 1), (2561, 2305, 130, 3), (2304, 2560, 96, 0)])
def test_large_products_leave_their_neighbours(B, dtype, M, N, K, col):
    """Products on pairs of multiprocessors into columns [col, col + N) of wider rows, the first of them at any alignment: the values, and guard
    elements before, behind and between the rows."""
    out = torch.full((M + 2, N + 7), 5.0, dtype=dtype, device="cuda")
    product_case(B, M, N, K, None, out=out[1: M + 1, col: col + N])
    assert (out[0] == 5).all() and (out[M + 1] == 5).all() and (out[:, :col] == 5).all() and (out[:, col + N:] == 5).all()
