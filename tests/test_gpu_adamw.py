"""The AdamW step over a list of tensors against its formulas in 64 bits: types, lengths from zero on, unaligned tensors, several
pushes, fp32 and 8-bit states (decoded here from the definition of E4M3 and of the scale bytes), captured steps, refusals.

Tolerances.  fp32: the kernel forms m and v with two roundings each and p with at most eight (sum of K pushes: K + 1), one of
them a square root and one a division of relative error 2^-22 at most; everything is held to 2^-20 of the largest magnitude
involved.  Rounding to a storage type adds half a step: bf16 2^-8, 8-bit states less than one step (stochastic): 2^-3."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
F32 = 2.0 ** -20
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def e4m3(codes):
    c = codes.astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where(c >> 7, -v, v)


def decode8(codes, scales):
    n = codes.size
    return e4m3(codes) * np.repeat(np.exp2(scales.astype(np.float64) - 127), 32)[:n]


def mx_decode(codes, scales, n):
    c = np.stack([codes & 15, codes >> 4], 1).reshape(-1)[:n].astype(np.int64)
    return np.where(c >> 3, -1, 1) * GRID[c & 7] * np.repeat(np.exp2(scales.astype(np.float64) - 127), 32)[:n]


def reference(p, m, v, gs, lr, t, decay, b1=0.9, b2=0.999, eps=1e-8, scale=1.0):
    g = scale * sum(gs) / len(gs)
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps), m, v


class Case:
    """Tensors of given lengths as views of flat buffers, with guard elements between and behind them."""

    def __init__(self, B, sizes, p_type, g_type, K, bits, gap=0, seed=0, shadow=False, decay=0.1, n_pushes=None):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits, self.K, self.decay, self.g_type = sizes, bits, K, decay, g_type
        step = 32 if gap == 0 else 1
        offs, at = [], gap
        for n in sizes:
            offs.append(at)
            at += -(-n // step) * step + gap
        self.offs, total = offs, -(-(at + 64) // 32) * 32
        dev = "cuda"
        self.flat_p = torch.from_numpy(rng.standard_normal(total) * 0.1).to(dev).to(p_type)
        def views(t, per=1):
            return [t[o // per: o // per + -(-n // per)] for o, n in zip(offs, sizes)]
        self.views = views
        self.flat_g, self.pushes = [], []
        for _ in range(n_pushes or K):
            g = torch.from_numpy(rng.standard_normal(total) * 1e-2).to(dev)
            if g_type == "mx":
                codes = torch.from_numpy(rng.integers(0, 256, total // 2 + 64, dtype=np.uint8)).to(dev)
                scales = torch.from_numpy(rng.integers(110, 124, total // 32 + 1, dtype=np.uint8)).to(dev)
                self.flat_g.append((codes, scales))
                self.pushes.append([B.MxTensor(a, b, 1, n, "linear") for a, b, n in zip(views(codes, 2), views(scales, 32), sizes)])
            else:
                g = g.to(g_type)
                self.flat_g.append(g)
                self.pushes.append(views(g))
        self.flat_shadow = torch.full((total,), 7.0, dtype=torch.bfloat16, device=dev) if shadow else None
        if bits == 32:
            self.flat = {"m": torch.from_numpy(rng.standard_normal(total) * 1e-2).float().to(dev),
                         "v": torch.from_numpy(rng.random(total) * 1e-4).float().to(dev)}
            self.state = {k: views(t) for k, t in self.flat.items()}
        else:
            # codes below 0x7F: all finite; m signed
            self.flat = {"m": torch.from_numpy((rng.integers(0, 127, total) | (rng.integers(0, 2, total) << 7)).astype(np.uint8)).to(dev),
                         "v": torch.from_numpy(rng.integers(0, 127, total).astype(np.uint8)).to(dev)}
            sc = total if gap else total // 32 + 1
            self.flat["m_scale"] = torch.from_numpy(rng.integers(108, 114, sc, dtype=np.uint8)).to(dev)
            self.flat["v_scale"] = torch.from_numpy(rng.integers(108, 114, sc, dtype=np.uint8)).to(dev)
            if gap:
                self.state = {k: views(self.flat[k]) for k in ("m", "v")}
                self.state |= {k: [self.flat[k][o: o + -(-n // 32)] for o, n in zip(offs, sizes)] for k in ("m_scale", "v_scale")}
            else:
                self.state = {k: views(t, 32 if "scale" in k else 1) for k, t in self.flat.items()}
        self.opt = B.AdamW(views(self.flat_p), self.pushes, weight_decay=decay, state_bits=bits, state=self.state, seed=77,
                           shadow=views(self.flat_shadow) if shadow else None)

    def numpy_grad(self, l, i):
        if self.g_type == "mx":
            q = self.pushes[l][i]
            return mx_decode(q.codes.cpu().numpy(), q.scales.cpu().numpy(), self.sizes[i])
        return self.pushes[l][i].double().cpu().numpy()

    def snapshot(self):
        out = []
        for i, n in enumerate(self.sizes):
            s = {k: self.state[k][i].cpu().numpy().copy() for k in self.state}
            if self.bits == 8:
                m, r = decode8(s["m"], s["m_scale"]), decode8(s["v"], s["v_scale"])
                s = {"m": m, "v": r * r}
            out.append((self.opt.params[i].double().cpu().numpy().copy(), s["m"].astype(np.float64), s["v"].astype(np.float64)))
        return out

    def check(self, before, lr, t, scale=1.0):
        for i, n in enumerate(self.sizes):
            if n == 0:
                continue
            p0, m0, v0 = before[i]
            p, m, v = reference(p0, m0, v0, [self.numpy_grad(l, i) for l in range(self.K)], lr, t, self.decay, scale=scale)
            got = self.opt.params[i].double().cpu().numpy()
            gm = sum(np.abs(self.numpy_grad(l, i)) for l in range(self.K)) / self.K * abs(scale)
            # the step without cancellation inside m: what its roundings are relative to
            top = lr * (0.9 * np.abs(m0) + 0.1 * gm) / (1 - 0.9 ** t) / (np.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
            # pushes that cancel: their mean g is off by d <= K 2^-24 gm, however small it is, so v = b2 v0 + c2 g^2 is off by
            # 2 c2 |g| d and sqrt(v) by the fraction c2 |g| d / v (with v0 = 0, |g| << gm: far more than 2^-20)
            g = np.abs(scale * sum(self.numpy_grad(l, i) for l in range(self.K))) / self.K
            top = np.abs(p0) + top * (1 + 0.001 * g * gm / np.maximum(v, 1e-300))
            tol = F32 * top + (2.0 ** -8 * np.abs(p) if self.opt.params[i].dtype == torch.bfloat16 else 0)
            assert np.all(np.abs(got - p) <= tol), ("p", i, n, np.abs(got - p).max())
            if self.flat_shadow is not None:
                sh = self.opt.shadow[i].double().cpu().numpy()
                assert np.array_equal(sh, self.opt.params[i].to(torch.bfloat16).double().cpu().numpy()), ("shadow", i)
            s = {k: self.state[k][i].cpu().numpy() for k in self.state}
            if self.bits == 32:
                assert np.all(np.abs(s["m"] - m) <= F32 * (np.abs(m0) + gm + 1e-30)), ("m", i)
                assert np.all(np.abs(s["v"] - v) <= F32 * (v0 + gm * gm + 1e-30)), ("v", i)
            else:
                r = np.sqrt(v)
                for name, want, got8 in (("m", m, decode8(s["m"], s["m_scale"])), ("v", r, decode8(s["v"], s["v_scale"]))):
                    blocks = np.abs(np.pad(want, (0, -n % 32))).reshape(-1, 32).max(1)
                    k = np.repeat(s[name + "_scale"].astype(np.float64) - 127, 32)[:n]
                    need = np.repeat(blocks, 32)[:n]
                    # least power of two with the block's top at most 448 of it (an fp32 rounding either way at the border)
                    assert np.all(need <= 448 * np.exp2(k) * (1 + F32)) and np.all((need > 224 * np.exp2(k) * (1 - F32)) | (k == -127)), (name, i)
                    a = np.abs(want) / np.exp2(k)
                    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(a, 1e-300))), -6) - 3)
                    off = np.abs(got8 - want) / np.exp2(k)
                    assert np.all(off <= step * (1 + 2.0 ** -10) + F32 * 448), (name, i, off.max())
                    if name == "v":
                        assert np.all(got8[want > 0] > 0), "a positive root must stay positive"


TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16),
         (torch.bfloat16, torch.float32), (torch.float32, "mx"), (torch.bfloat16, "mx")]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_type,g_type", TYPES)
@pytest.mark.parametrize("K", [1, 3])
def test_step_matches_the_formulas(B, bits, p_type, g_type, K):
    c = Case(B, [1, 0, 7, 8, 31, 32, 33, 2047, 2048, 2049, 5000, 40001], p_type, g_type, K, bits, shadow=p_type == torch.float32, seed=K)
    for t in (1, 2, 1000):
        before = c.snapshot()
        c.opt.step(t, 3e-3, grad_scale=0.5)
        torch.cuda.synchronize()
        c.check(before, float(np.float32(3e-3)), t, 0.5)
    c.opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_type,g_type", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_unaligned_tensors_and_their_neighbours(B, bits, p_type, g_type):
    """Tensors one element apart: no access is 16-byte aligned, and what lies between the tensors stays as it was."""
    c = Case(B, [1, 7, 33, 2049, 300, 5], p_type, g_type, 2, bits, gap=1, seed=5)
    marks = torch.ones(c.flat_p.numel(), dtype=torch.bool)
    for o, n in zip(c.offs, c.sizes):
        marks[o: o + n] = False
    old = [t.clone() for t in (c.flat_p, c.flat["m"], c.flat["v"])]
    before = c.snapshot()
    c.opt.step(3, 1e-3)
    torch.cuda.synchronize()
    c.check(before, float(np.float32(1e-3)), 3)
    for a, b in zip(old, (c.flat_p, c.flat["m"], c.flat["v"])):
        assert torch.equal(a.cpu()[marks], b.cpu()[marks])
        assert not torch.equal(a, b)


def test_first_pushes_only(B):
    """K = 2 of four bound pushes: the mean of the first two."""
    c = Case(B, [513, 64], torch.float32, torch.float32, 2, 32, n_pushes=4)
    before = c.snapshot()
    c.opt.step(1, 1e-3, K=2)
    torch.cuda.synchronize()
    c.check(before, float(np.float32(1e-3)), 1)


def test_eight_bit_states_are_unbiased_and_decay(B):
    """With zero gradients v decays by 1 - b2 a step, far below half an 8-bit step: on average over many elements the stored root
    has to follow it.  65536 elements, 200 steps: the mean of r must be (0.999)^100 of the start; one rounding's relative
    deviation is under 2^-3 / sqrt(12) an element, so the mean of 65536 elements over 200 steps deviates by about
    sqrt(200) 2^-3 / sqrt(12) / 256 = 0.002: five of those."""
    n = 65536
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt = B.AdamW([p], [[g]], state_bits=8, seed=3, weight_decay=0.0)
    g.fill_(1.0)
    opt.step(1, 0.0)
    g.zero_()
    r0 = decode8(opt.state["v"][0].cpu().numpy(), opt.state["v_scale"][0].cpu().numpy()).mean()
    for t in range(2, 202):
        opt.step(t, 0.0)
    r = decode8(opt.state["v"][0].cpu().numpy(), opt.state["v_scale"][0].cpu().numpy()).mean()
    assert abs(r / r0 / 0.999 ** 100 - 1) < 0.01
    assert not p.any()


def test_same_calls_give_the_same_bits_in_any_list(B):
    """Stochastic rounding goes by seed, step, index in the list and element: a longer list behind a tensor changes nothing."""
    outs = []
    for extra in (0, 3):
        torch.manual_seed(0)
        ps = [torch.randn(10007, device="cuda")] + [torch.randn(999, device="cuda") for _ in range(extra)]
        gs = [torch.ones_like(p) * 0.01 for p in ps]
        opt = B.AdamW(ps, [gs], state_bits=8, seed=9)
        for t in (1, 2, 3):
            opt.step(t, 1e-3)
        outs.append([ps[0].cpu()] + [opt.state[k][0].cpu() for k in ("m", "v", "m_scale", "v_scale")])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_captured_steps_and_another_stream(B):
    """Steps replayed from a graph, step number and learning rate on the device, equal steps called one by one; the same on a
    stream that is not the current one."""
    def fresh():
        torch.manual_seed(1)
        ps = [torch.randn(3001, device="cuda"), torch.randn(64, device="cuda").bfloat16()]
        gs = [torch.randn(3001, device="cuda"), torch.randn(64, device="cuda")]
        return ps, B.AdamW(ps, [gs], state_bits=8, seed=4)
    ps, opt = fresh()
    for t in range(1, 6):
        opt.step(t, 1e-2 * t)
    want = [p.clone() for p in ps] + [s.clone() for k in opt.state for s in opt.state[k]]
    ps, opt = fresh()
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step.add_(1)
        opt.step(step, lr)
    for t in range(1, 6):
        lr.fill_(1e-2 * t)
        g.replay()
    torch.cuda.synchronize()
    assert step.item() == 5
    assert all(torch.equal(a, b) for a, b in zip(want, ps + [s for k in opt.state for s in opt.state[k]]))
    del g
    ps, opt = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in range(1, 6):
        opt.step(t, 1e-2 * t, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, ps + [s for k in opt.state for s in opt.state[k]]))


def test_a_handle_dropped_during_a_capture(B):
    """Freeing one handle's tables leaves another's capture whole."""
    p, g = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    opt, other = B.AdamW([p], [[g]], weight_decay=0.0), B.AdamW([torch.ones(10, device="cuda")], [[torch.ones(10, device="cuda")]])
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.full((1,), 0.5, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        other.close()
        opt.step(step, lr)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.allclose(p, torch.full_like(p, 0.5), rtol=2.0 ** -18)       # m / sqrt(v) = 1 up to eps


def test_the_first_step_on_another_stream(B):
    """A list is ready for any stream when it has been made, the zeros of its states too."""
    side, n = torch.cuda.Stream(), 1 << 22
    p, g = torch.ones(n, device="cuda"), torch.ones(n, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    opt = B.AdamW([p], [[g]], weight_decay=0.0)
    opt.step(1, 0.5, stream=side)
    torch.cuda.synchronize()
    assert torch.allclose(opt.state["m"][0], torch.full_like(p, 0.1), rtol=2.0 ** -22)
    assert torch.allclose(p, torch.full_like(p, 0.5), rtol=2.0 ** -18)


def test_non_finite_gradients_show(B):
    p, g = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    g[3] = float("nan")
    g[40] = float("inf")
    opt = B.AdamW([p], [[g]])
    opt.step(1, 1e-3)
    assert torch.isnan(p).nonzero().flatten().tolist() == [3, 40]      # inf / inf
    p2 = torch.ones(96, device="cuda")
    g2 = torch.ones(96, device="cuda")
    g2[3] = float("nan")
    opt = B.AdamW([p2], [[g2]], state_bits=8)
    opt.step(1, 1e-3)
    assert opt.state["m_scale"][0].cpu().tolist()[0] == 255 and opt.state["m_scale"][0].cpu().tolist()[1] < 255
    g2[3] = 1.0
    opt.step(2, 1e-3)
    assert torch.isnan(p2[:32]).all() and not torch.isnan(p2[32:]).any()


def test_refusals_on_the_device(B):
    p, g = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    opt = B.AdamW([p], [[g]])
    for args, kw in (((0, 1e-3), {}), ((1 << 32, 1e-3), {}), ((1, -1.0), {}), ((1, float("nan")), {}), ((1, 1e-3), {"K": 2}), ((1, 1e-3), {"K": 0}),
                     ((1, 1e-3), {"grad_scale": float("inf")})):
        with pytest.raises(B.SimError) as e:
            opt.step(*args, **kw)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        opt.step(torch.ones(1, dtype=torch.int64, device="cuda"), 1e-3)
    for kw in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0), dict(eps=1e-60), dict(weight_decay=-1.0)):
        with pytest.raises(B.SimError) as e:
            B.AdamW([p], [[g]], **kw)
        assert e.value.status == 1
    for ps, gs, kw in (([p], [[g[:7]]], {}), ([p], [[g.int()]], {}), ([p.half()], [[g]], {}), ([p], [], {}), ([p, p], [[g]], {}), ([p], [[g.cpu()]], {}),
                       ([p], [[g]], dict(state_bits=16)), ([p], [[g]], dict(state={"m": [g]})), ([p[::2]], [[g[:4]]], {}),
                       ([p.bfloat16()], [[g]], dict(shadow=[g])), ([p], [[g]], dict(weight_decay=[0.1, 0.2]))):
        with pytest.raises(ValueError):
            B.AdamW(ps, gs, **kw)
    assert not p.any()


def test_overlapping_buffers_are_refused(B):
    """The same parameter twice, states shared by two parameters, a gradient inside another parameter; two pushes may be one buffer."""
    p, g = torch.zeros(256, device="cuda"), torch.ones(256, device="cuda")
    q = torch.zeros(256, device="cuda")
    z = lambda: torch.zeros(256, device="cuda")  # noqa: E731
    m = z()
    for ps, gs, state in (([p, p], [g, g], None), ([p, q], [g, g], {"m": [m, m], "v": [z(), z()]}), ([p, q], [g, p], None), ([p[:200], p[199:]], [g[:200], g[199:]], None)):
        with pytest.raises(B.SimError) as e:
            B.AdamW(ps, [gs], state=state)
        assert e.value.status == 1 and "overlaps" in str(e.value)
    opt = B.AdamW([p], [[g], [g]], weight_decay=0.0)
    opt.step(1, 0.5)
    assert torch.allclose(p, torch.full_like(p, -0.5), rtol=2.0 ** -19)      # m / sqrt(v) = 1 up to eps


def test_offsets_beyond_32_bits(B):
    """2^31 + 5000 elements, bf16 parameters: the last elements, and those around element 2^31, move as the formulas say."""
    n = (1 << 31) + 5000
    p, g = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda"), torch.full((n,), 0.25, dtype=torch.bfloat16, device="cuda")
    g[-1], g[1 << 31] = -0.125, 0.0
    opt = B.AdamW([p], [[g]], state_bits=8, weight_decay=0.0, seed=1)
    opt.step(1, 0.25)
    # first step: m / (1 - b1) = g, sqrt(v / (1 - b2)) = |g|: p moves by the step size against the sign of g
    at = torch.tensor([0, 12345, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, n - 2, n - 1], device="cuda")
    assert p[at].float().cpu().tolist() == [0.25, 0.25, 0.25, 0.5, 0.25, 0.25, 0.75]
    blocks = opt.state["v_scale"][0]
    assert blocks.numel() == (n + 31) // 32 and (blocks != 0).all()
    del opt, p, g
    torch.cuda.empty_cache()
