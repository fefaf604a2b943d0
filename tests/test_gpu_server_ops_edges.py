"""The server's operators where their ranges end: moments next to the smallest fp32 numbers, unaligned lists of every push type, the documented
rounding of 8-bit states bit for bit, results between guard elements, long waits and small data sets.  Tolerances are derived in each test."""
import time

import numpy as np
import pytest
import torch

from parity import to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def tiny(n, seed):
    """Gradients of 2^-62 to 2^-57: their squares times 1 - b2 = 2^-10 lie on both sides of 2^-126."""
    rng = np.random.default_rng(seed)
    return (np.exp2(rng.uniform(-62, -57, n)) * rng.choice([-1.0, 1.0], n)).astype(np.float32)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("at", [0, 1])
def test_second_moments_under_the_smallest_normal(B, bits, at):
    """With eps = 1e-20 the divisor is |g| for gradients far above eps, however small their squares.  v is formed in fp32: under 2^-126 it is off by
    up to 2^-150, half a step there (its own rounding; s2 g is a normal number), so its root by the fraction 2^-151 / v; the rest as
    elsewhere 2^-20.  at = 1: unaligned."""
    n, eps, lr = 4500, 1e-20, 0.5
    g = tiny(n, 3)
    flat = [torch.zeros(n + 8, device="cuda") for _ in range(2)]
    p, grad = (t[at: at + n] for t in flat)
    grad.copy_(torch.from_numpy(g))
    opt = B.AdamW([p], [[grad]], eps=eps, weight_decay=0.0, state_bits=bits)
    opt.step(1, lr)
    g64 = g.astype(np.float64)
    want, v = -lr * g64 / (np.abs(g64) + eps), 0.001 * g64 * g64
    got = p.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= lr * (2.0 ** -20 + 2.0 ** -151 / v))
    if bits == 8:
        assert bool((opt.state["v"][0] != 0).all())
        return
    m0, v0 = (opt.state[k][0].double().cpu().numpy() for k in ("m", "v"))
    assert np.all(np.abs(v0 - v) <= 2.0 ** -20 * v + 2.0 ** -150)
    opt.step(2, lr)
    m, v = 0.9 * m0 + 0.1 * g64, 0.999 * v0 + 0.001 * g64 * g64
    want = got - lr * (m / (1 - 0.9 ** 2)) / (np.sqrt(v / (1 - 0.999 ** 2)) + eps)
    # v' = fma(b2, v, rn(s s)), s = s2 g, has two roundings (with v = 0 the sum was exact): up to 2 x 2^-150, so 2^-150 / v of the root
    assert np.all(np.abs(p.double().cpu().numpy() - want) <= 2.0 ** -20 * (np.abs(got) + lr) + lr * 2.0 ** -150 / v)


def test_second_moments_under_the_smallest_normal_of_the_simulated_server(B):
    """The same in the simulated server's update: one row x, y = 1, w = 0, so the first gradient is -x exactly."""
    d, eps, eta = 256, 1e-20, 0.5
    x = tiny(d, 4)
    data = {"model": "lsq", "X": x[None], "y": np.ones(1, np.float32), "n_classes": 1, "hidden": 0}
    sim = B.Simulation(to_device(data), P=1, K=1, variant="ksync", delay_kind="exp", mu=1.0, eta=eta, m=1, seed=0, n_replicas=2)
    sim.set_adamw((0.9, 0.999), eps, 0.0)
    sim.set_params(torch.zeros(d, device="cuda"))
    sim.run(1)
    g = -x.astype(np.float64)
    for w in sim.params():
        assert np.all(np.abs(w - -eta * g / (np.abs(g) + eps)) <= eta * (2.0 ** -20 + 2.0 ** -151 / (0.001 * g * g)))
    sim.close()


def test_the_simulated_server_refuses_eps_whose_reciprocal_is_no_normal_number(B):
    data = {"model": "lsq", "X": np.ones((4, 8), np.float32), "y": np.ones(4, np.float32), "n_classes": 1, "hidden": 0}
    sim = B.Simulation(to_device(data), P=1, K=1, variant="ksync", delay_kind="exp", mu=1.0, eta=0.1, m=1, seed=0, n_replicas=1)
    for eps in (2.0 ** -127, 2.0 ** 126, 1e300):
        with pytest.raises(B.SimError) as e:
            sim.set_adamw(eps=eps)
        assert e.value.status == 1
    sim.close()


def test_a_wait_with_a_limit_in_time_keeps_to_it(B):
    """The self-test's second wait sleeps on a barrier that nobody arrives at and gives up after 50 ms by the clock, however often the hardware
    wakes it; the wait for a tile of a large product is this one with four seconds."""
    data = {"model": "lsq", "X": np.ones((4, 8), np.float32), "y": np.ones(4, np.float32), "n_classes": 1, "hidden": 0}
    sim = B.Simulation(to_device(data), P=1, K=1, variant="ksync", delay_kind="exp", mu=1.0, eta=0.1, m=1, seed=0, n_replicas=1)
    torch.cuda.synchronize()
    begin = time.perf_counter()
    sim.selftest_wait_timeout()
    torch.cuda.synchronize()
    took = time.perf_counter() - begin
    with pytest.raises(B.SimError) as e:
        sim.trace_size()
    assert e.value.status == 4
    sim.close()
    assert 0.05 <= took < 0.5


def test_the_risk_in_mxfp4_of_a_small_data_set_takes_little_memory(B):
    """The logits of 1024 replicas over 2001 rows are 8 MB; with everything else the first call's buffers stay under 32 MB (cudaMalloc rounds
    up to 2 MB).  The value is that of the same replicas in smaller groups."""
    rng = np.random.default_rng(6)
    data = {"model": "lsq", "X": rng.standard_normal((2001, 16)).astype(np.float32), "y": rng.standard_normal(2001).astype(np.float32), "n_classes": 1, "hidden": 0}
    dev, kw = to_device(data), dict(P=2, K=1, variant="ksync", delay_kind="exp", mu=1.0, eta=0.1, m=4, seed=1)
    warm = B.Simulation(dev, n_replicas=1, **kw)               # kernels are loaded, torch has its memory
    warm.run(1)
    warm.eval_loss(mxfp4=True)
    sim = B.Simulation(dev, n_replicas=1024, **kw)
    sim.run(7)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    got = sim.eval_loss(mxfp4=True)
    assert free - torch.cuda.mem_get_info()[0] < 32 << 20
    for base in (0, 1019):
        part = B.Simulation(dev, n_replicas=5, replica_base=base, **kw)
        part.run(7)
        # other tiles, so other orders of the 16 sums of the logits: each within 16 x 2^-23 of its magnitude, doubled by the square
        assert np.allclose(part.eval_loss(mxfp4=True), got[base: base + 5], rtol=2.0 ** -16, atol=0)
        part.close()
    sim.close()
    warm.close()
