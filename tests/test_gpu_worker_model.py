"""The worker's operators in use: log probabilities of the simulated softmax and MLP models' samples, and a worker's step (forward pass with activations kept
in 8 bits, loss, backward pass, push in MXFP4, AdamW) as one run.

Log probabilities against the oracle's arithmetic in 64 bits: softmax 1e-5 of the logits' magnitude (an fp32 sum of d terms, 32 lanes: (d / 32 + 5) 2^-24 of the
sum of magnitudes, which is below 1e-5 for these d), MLP 1e-3 (the bound that its risk has)."""
import numpy as np
import pytest
import torch

from oracle import models
from paper_2003_10579_b200 import inputs
from parity import to_device
from worker_ref import act, f64, slope, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("model,variant,n,d,C,H", [("softmax", "ksync", 1500, 200, 10, 0), ("softmax", "kbatchasync", 777, 64, 3, 0), ("softmax", "kasync", 300, 128, 16, 0),
                                                   ("mlp2", "kasync", 1000, 128, 3, 64), ("mlp2", "ksync", 2049, 256, 10, 192)])
def test_log_probabilities_of_samples(model, variant, n, d, C, H):
    from paper_2003_10579_b200 import binding as B
    data = inputs.make_mixture(n, d, C, 0.3, 33, *(("mlp2", H) if H else ()))
    sim = B.Simulation(to_device(data), P=4, K=2, variant=variant, delay_kind="exp", mu=1.0, eta=0.02, m=128 if H else 8, seed=1, n_replicas=3)
    if H:
        sim.set_params(torch.from_numpy(inputs.mlp_init(d, H, C, 37)).cuda())
    for steps in (0, 7):
        if steps:
            sim.run(steps)
        risk, w = sim.eval_loss(), sim.params().astype(np.float64)
        for r, first, rows in ((0, 0, None), (2, 5, n - 9), (1, n - 1, 1), (1, n, 0)):
            got = sim.log_probs(r, first, rows, top=min(3, C))
            rows = n - first if rows is None else rows
            X, y = data["X"][first:first + rows], data["y"][first:first + rows].astype(np.int64)
            if H:
                o1, o2, o3 = d * H, d * H + H, d * H + H + H * C
                h = np.maximum(models.bf16_round(X) @ models.bf16_round(w[r][:o1].reshape(d, H)) + w[r][o1:o2], 0.0)
                z = h @ w[r][o2:o3].reshape(H, C) + w[r][o3:]
            else:
                z = X.astype(np.float64) @ w[r].reshape(C, d).T
            tol = (1e-3 if H else 1e-5) * (1 + np.abs(z).max(initial=0.0))
            lp = z - z.max(1, keepdims=True, initial=-np.inf)
            lp = lp - np.log(np.exp(lp).sum(1, keepdims=True))
            assert got["logp"].shape == (rows,) and np.abs(got["logp"] - lp[np.arange(rows), y]).max(initial=0.0) <= 2 * tol
            assert np.abs(got["entropy"] + (np.exp(lp) * lp).sum(1)).max(initial=0.0) <= 10 * tol
            # the classes come in an order that the exact values allow: each at most a rounding below the one before
            ranked = np.take_along_axis(lp, got["top_ids"].astype(np.int64), 1)
            assert np.abs(got["top_logp"] - ranked).max(initial=0.0) <= 2 * tol and (np.diff(ranked, axis=1) <= 2 * tol).all()
            if rows == n:
                assert abs(-got["logp"].mean(dtype=np.float64) - risk[r]) <= 2 * tol
    for bad in (dict(replica=3), dict(replica=-1), dict(first=n + 1, rows=0), dict(first=0, rows=n + 1), dict(top=C + 1)):
        with pytest.raises(B.SimError):
            sim.log_probs(**bad)
    sim.close()


def test_log_probabilities_need_classes():
    from paper_2003_10579_b200 import binding as B
    data = inputs.make_lsq(100, 64, 0.1, 31)
    sim = B.Simulation(to_device(data), P=4, K=2, variant="ksync", delay_kind="exp", mu=1.0, eta=0.02, m=8, seed=1, n_replicas=2)
    with pytest.raises(B.SimError):
        sim.log_probs()
    sim.close()


def run_worker(B, p, x, tokens, act_name):
    """Loss of one step of a residual block and a vocabulary head, and its gradients, with nothing but the 8-bit forms kept between the passes."""
    x8 = B.checkpoint(x)
    h, z8 = B.linear(x, p["w1"], p["b1"], act=act_name, keep=True)
    y = B.linear(h, p["w2"], p["b2"], residual=x)
    del h
    logits = B.linear(y, p["head"])
    n = int((tokens >= 0).sum())
    lp = B.log_probs(logits, tokens, top=2, d_logp=torch.full((x.shape[0],), -1.0 / n, device="cuda"), d_entropy=torch.full((x.shape[0],), -0.01, device="cuda"), out=logits)
    y8 = B.checkpoint(y)
    dy, dhead, _ = B.linear_backward(lp.dlogits, y8, p["head"], need="xw")
    dz, dw2, db2 = B.linear_backward(dy, z8, p["w2"], x_act=act_name)
    dx, dw1, db1 = B.linear_backward(dz, x8, p["w1"], residual=dy)
    loss = -lp.logp.sum() / n - 0.01 * lp.entropy.sum()
    return loss, {"w1": dw1, "b1": db1, "w2": dw2, "b2": db2, "head": dhead}, dx, (z8, x8, y8)


@pytest.mark.parametrize("T,d,f,V", [(50, 96, 200, 3000), (7, 33, 65, 501)])
def test_a_workers_step_and_its_push(T, d, f, V):
    """The gradient that the step computes is the loss' in 64 bits, differentiated where the kept values stand; pushed in MXFP4 through AdamW it moves the parameters the
    way the server's own tests hold."""
    from paper_2003_10579_b200 import binding as B
    gen = torch.Generator(device="cuda").manual_seed(T)
    rnd = lambda *s, k=1.0, dt=torch.bfloat16: (torch.randn(*s, generator=gen, device="cuda") * k).to(dt)  # noqa: E731
    p = {"w1": rnd(f, d, k=d**-0.5), "b1": rnd(f, k=0.1, dt=torch.float32), "w2": rnd(d, f, k=f**-0.5), "b2": rnd(d, k=0.1, dt=torch.float32), "head": rnd(V, d, k=d**-0.5)}
    x, tokens = rnd(T, d), torch.randint(-1, V, (T,), generator=gen, device="cuda")
    tokens[0] = 3
    loss, grads, dx, (z8, x8, y8) = run_worker(B, p, x, tokens, "gelu")
    P = {k: f64(v) for k, v in p.items()}
    X, t = f64(x), tokens.cpu().numpy()
    Z, X8, Y8 = values(z8)[0], values(x8)[0], values(y8)[0]
    h = act("gelu", X @ P["w1"].T + P["b1"])
    y = h @ P["w2"].T + P["b2"] + X
    l = y @ P["head"].T
    lp = l - np.log(np.exp(l).sum(1, keepdims=True))
    pr, ent = np.exp(lp), -(np.exp(lp) * lp).sum(1)
    n = (t >= 0).sum()
    want = -lp[np.arange(T), t][t >= 0].sum() / n - 0.01 * ent.sum()
    assert abs(float(loss) - want) <= 0.01 * abs(want)                    # bf16 activations and logits: 2^-8 each along three products
    g = np.where(t >= 0, -1.0 / n, 0.0)
    dl = -pr * (g[:, None] - 0.01 * (lp + ent[:, None]))
    dl[np.arange(T)[t >= 0], t[t >= 0]] += g[t >= 0]
    dy = dl @ P["head"]
    dz = (dy @ P["w2"]) * slope("gelu", Z)
    ref = {"head": dl.T @ Y8, "w2": dy.T @ act("gelu", Z), "b2": dy.sum(0), "w1": dz.T @ X8, "b1": dz.sum(0)}
    for k, v in list(ref.items()) + [("dx", dz @ P["w1"] + dy)]:
        got = f64(dx if k == "dx" else grads[k])
        # every stage rounds to 16 bits (2^-8 of its elements, a few stages deep, partly averaged out)
        assert np.linalg.norm(got - v) <= 0.02 * np.linalg.norm(v), (k, np.linalg.norm(got - v) / np.linalg.norm(v))

    # the same step into push buffers that stay: two pushes in 4 bits, averaged by the server's AdamW
    names = list(grads)
    shapes = {k: grads[k].shape for k in names}
    pushes = [[B.mx_quantize(grads[k].reshape(-1), layout="linear", rounding="stochastic", seed=s) for k in names] for s in (1, 2)]
    master = [p[k].float().reshape(-1).clone() for k in names]
    before = [m.clone() for m in master]
    opt = B.AdamW(master, pushes, weight_decay=0.0)
    opt.step(1, 1e-3)
    for k, m, b, q in zip(names, master, before, zip(*pushes)):
        mean = sum(B.mx_dequantize(v).reshape(-1) for v in q) / 2
        moved = m - b
        live = mean.abs() > 1e-5
        torch.testing.assert_close(moved[live], -1e-3 * torch.sign(mean[live]), rtol=2e-3, atol=1e-6)      # the first step: m / sqrt(v) is the sign, eps 1e-8 beside 1e-5
        assert moved.numel() == int(np.prod(shapes[k]))


def test_a_workers_step_captured_and_replayed():
    """A step captured into a graph gives the eager step's bits, on new data too."""
    from paper_2003_10579_b200 import binding as B
    gen = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s, k=1.0, dt=torch.bfloat16: (torch.randn(*s, generator=gen, device="cuda") * k).to(dt)  # noqa: E731
    T, d, f, V = 200, 120, 333, 2001
    p = {"w1": rnd(f, d, k=d**-0.5), "b1": rnd(f, k=0.1, dt=torch.float32), "w2": rnd(d, f, k=f**-0.5), "b2": rnd(d, k=0.1, dt=torch.float32), "head": rnd(V, d, k=d**-0.5)}
    x, tokens = rnd(T, d), torch.randint(0, V, (T,), generator=gen, device="cuda")
    n = torch.full((T,), -1.0 / T, device="cuda")

    def step():
        h, z8 = B.linear(x, p["w1"], p["b1"], act="silu", keep=True)
        y = B.linear(h, p["w2"], p["b2"], residual=x)
        logits = B.linear(y, p["head"])
        lp = B.log_probs(logits, tokens, d_logp=n, out=logits)
        dy, dhead, _ = B.linear_backward(lp.dlogits, B.checkpoint(y), p["head"], need="xw")
        dz, dw2, db2 = B.linear_backward(dy, z8, p["w2"], x_act="silu")
        return [lp.logp, dhead, dw2, db2, *B.linear_backward(dz, B.checkpoint(x), p["w1"], residual=dy)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(2):
        x.copy_(rnd(T, d))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_results_on_the_handles_stream_wait_for_the_current_one():
    """A handle with a stream of its own writes its results into new memory, which the current stream may still be reading as another tensor that was let go."""
    from paper_2003_10579_b200 import binding as B
    n, d, C = 4096, 64, 10
    data = inputs.make_mixture(n, d, C, 0.3, 33)
    st = torch.cuda.Stream()
    sim = B.Simulation(to_device(data), P=4, K=2, variant="ksync", delay_kind="exp", mu=1.0, eta=0.02, m=8, seed=1, n_replicas=3, stream=st)
    sim.run(2)
    want = sim.log_probs()
    for call in (sim.log_probs, sim.eval_loss, sim.params, sim.trace):
        old = [torch.full((n,), 7.0, device="cuda") for _ in range(4)] + [torch.full((3, sim.n_params), 7.0, device="cuda"), torch.full((3,), 7.0, device="cuda")]
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)                    # some 10 ms
        kept = [t.clone() for t in old]
        del old
        call()
        torch.cuda.synchronize()
        assert all((t == 7.0).all() for t in kept), call
    got = sim.log_probs()
    assert all((got[k] == want[k]).all() for k in want)
    sim.close()
