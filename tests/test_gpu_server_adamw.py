"""The simulated parameter server with AdamW as its update, against the oracle (schedule bit-exact, parameters to 1e-5 relative,
losses to 1e-5 relative, as for the plain step), and the full-data risk with data and parameters in MXFP4."""
import numpy as np
import pytest
import torch

from oracle import core
from oracle.sim import OracleReplica
from paper_2003_10579_b200 import inputs
from parity import assert_loss_close, assert_params_close, assert_schedule_equal, to_device
from test_gpu_mx import quantise

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def simulate(B, data, *, chunks, adamw, w0, eta=0.01, R=3, base=0, K0=0, ti=0.0, **kw):
    sim = B.Simulation(to_device(data), eta=eta, n_replicas=R, replica_base=base, **kw)
    sim.set_adamw(adamw[:2], adamw[2], adamw[3])
    if ti > 0:
        sim.set_adasync(K0, ti)
    sim.set_params(torch.from_numpy(w0).cuda())
    snaps = []
    for c in chunks:
        sim.run(c)
        snaps.append(sim.params())
    tr = sim.trace()
    sim.close()
    return snaps, tr


@pytest.mark.parametrize("variant", list(core.VARIANTS))
@pytest.mark.parametrize("model,d,m,K,P,R", [("lsq", 64, 16, 2, 4, 3), ("lsq", 1000, 9, 3, 5, 3), ("logistic", 516, 6, 4, 8, 3), ("lsq", 2052, 4, 1, 3, 3),
                                             ("logistic", 4096, 5, 2, 3, 2), ("lsq", 5000, 3, 2, 4, 2), ("lsq", 1024, 8, 3, 4, 300), ("logistic", 100, 7, 2, 3, 300)])
def test_adamw_server_matches_the_oracle(B, variant, model, d, m, K, P, R):
    """Every block shape of the linear kernel (rows up to 8192 features, few and many replicas), ragged tiles, all variants."""
    data = inputs.make_lsq(2000, d, 0.5, 91) if model == "lsq" else inputs.make_logistic(2000, d, 0.1, 92)
    w0 = np.random.default_rng(3).standard_normal(d).astype(np.float32)
    adamw, kw = (0.9, 0.99, 1e-6, 0.05), dict(P=P, K=K, variant=variant, delay_kind="shifted_exp", mu=1.0, shift=0.5, m=m, seed=4)
    chunks = [1, 1, 5, 13]
    snaps, tr = simulate(B, data, chunks=chunks, adamw=adamw, w0=w0, R=R, base=5, **kw)
    sched = core.BulkSchedule(variant, P, K, "shifted_exp", 1.0, 0.5, 4, R, replica_base=5).run(sum(chunks))
    assert_schedule_equal(tr, sched)
    for r in {0, R - 1}:
        o = OracleReplica(model=data["model"], X=data["X"], y=data["y"], w0=w0, eta=0.01, replica=5 + r, adamw=adamw, **kw)
        for c, w in zip(chunks, snaps):
            o.run(c)
            assert_params_close(w[r], o.w, "%s %s replica %d update %d" % (model, variant, r, o.j))
        assert_loss_close(tr["loss"][r], o.trace_arrays()["loss"], "%s %s" % (model, variant))


def test_growing_K_and_resume(B):
    """K changes on the way (the mean over K follows it); one run of 40 updates and runs of 1, 7 and 32 give the same bits."""
    data = inputs.make_lsq(1500, 256, 0.5, 93)
    w0 = np.random.default_rng(5).standard_normal(256).astype(np.float32)
    kw = dict(P=8, K=1, variant="kasync", delay_kind="exp", mu=1.0, m=6, seed=2, adamw=(0.9, 0.999, 1e-8, 0.0), w0=w0, K0=1, ti=4.0)
    (a,), ta = simulate(B, data, chunks=[40], **kw)
    snaps, tb = simulate(B, data, chunks=[1, 7, 32], **kw)
    assert np.array_equal(a, snaps[-1]) and all(np.array_equal(ta[k], tb[k]) for k in ta)
    assert len(set(ta["K"][0].tolist())) > 1
    o = OracleReplica(model="lsq", X=data["X"], y=data["y"], w0=w0, eta=0.01, replica=0, P=8, K=1, variant="kasync", delay_kind="exp", mu=1.0, m=6, seed=2, K0=1,
                      t_interval=4.0, adamw=(0.9, 0.999, 1e-8, 0.0)).run(40)
    assert_params_close(a[0], o.w, "growing K")


@pytest.mark.parametrize("variant", ["ksync", "kasync"])
def test_K_from_the_risk(B, variant):
    """K that follows the full-data risk of the AdamW server's parameters."""
    data = inputs.make_lsq(600, 32, 0.1, 94)
    w0 = np.zeros(32, np.float32)
    adamw, kw = (0.9, 0.999, 1e-8, 0.0), dict(P=6, K=1, variant=variant, delay_kind="exp", mu=1.0, m=8, seed=3)
    sim = B.Simulation(to_device(data), eta=0.05, n_replicas=2, **kw)
    sim.set_adamw(adamw[:2], adamw[2], adamw[3])
    sim.set_adasync_loss(1, 2.0)
    sim.set_params(torch.from_numpy(w0).cuda())
    sim.run(60)
    w, tr = sim.params(), sim.trace()
    sim.close()
    for r in range(2):
        o = OracleReplica(model="lsq", X=data["X"], y=data["y"], w0=w0, eta=0.05, replica=r, K0=1, t_interval=2.0, k_rule="loss", adamw=adamw, **kw).run(60)
        assert len(o.k_events) > 1 and o.trace["K"] == tr["K"][r].tolist()
        assert_params_close(w[r], o.w, "K from the risk, %s" % variant)


def test_adamw_server_equals_the_step_over_tensors(B):
    """The simulated server's update and the step over a list of tensors are one operator: with P = K = 1 and a data set of one
    row every minibatch is that row, so the gradients can be formed here and stepped with the other entry point."""
    d = 64
    g = torch.Generator().manual_seed(7)
    X, y = torch.randn(1, d, generator=g), torch.randn(1, generator=g)
    data = {"model": "lsq", "X": X.numpy(), "y": y.numpy(), "n_classes": 1, "hidden": 0}
    w0 = torch.randn(d, generator=g)
    snaps, _ = simulate(B, data, chunks=[1] * 6, adamw=(0.9, 0.99, 1e-8, 0.1), w0=w0.numpy(), eta=0.05, R=1, P=1, K=1, variant="ksync", delay_kind="exp", mu=1.0, m=1, seed=0)
    p, grad = w0.clone().cuda(), torch.zeros(d, device="cuda")
    opt = B.AdamW([p], [[grad]], betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    for t in range(6):
        grad.copy_((X[0].double() * (X[0].double() @ p.cpu().double() - y[0].double())).float())
        opt.step(t + 1, 0.05)
        # the gradients differ by the roundings of a 64-term dot product, and m / sqrt(v) passes that on once
        assert np.allclose(snaps[t][0], p.cpu().numpy(), rtol=0, atol=64 * 2.0 ** -22)


def test_adamw_refusals(B):
    kw = dict(P=2, K=1, variant="ksync", delay_kind="exp", mu=1.0, m=2, seed=0, n_replicas=1)
    lsq = to_device(inputs.make_lsq(50, 8, 0.1, 1))
    sim = B.Simulation(lsq, eta=0.1, **kw)
    for bad in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.5)), dict(eps=0.0), dict(eps=float("inf")), dict(weight_decay=-0.1), dict(weight_decay=float("nan"))):
        with pytest.raises(B.SimError) as e:
            sim.set_adamw(**bad)
        assert e.value.status == 1
    sim.run(1)
    with pytest.raises(B.SimError) as e:
        sim.set_adamw()
    assert e.value.status == 5
    sim.close()
    for data, eta in ((None, 0.1), (to_device(inputs.make_mixture(60, 8, 3, 0.5, 2)), 0.1), (lsq, -0.1)):
        sim = B.Simulation(data, eta=eta, **kw)
        with pytest.raises(B.SimError) as e:
            sim.set_adamw()
        assert e.value.status == 1
        sim.close()


@pytest.mark.parametrize("model,n,d,C,variant,R", [("lsq", 1000, 64, 1, "ksync", 3), ("lsq", 9001, 200, 1, "kbatchasync", 70), ("logistic", 2500, 520, 1, "kasync", 130),
                                                   ("softmax", 1500, 200, 10, "ksync", 20), ("softmax", 777, 64, 3, "kbatchasync", 5)])
def test_risk_in_mxfp4_matches_a_plain_evaluation(B, model, n, d, C, variant, R):
    if model == "lsq":
        data = inputs.make_lsq(n, d, 0.1, 31)
    elif model == "logistic":
        data = inputs.make_logistic(n, d, 0.05, 32)
    else:
        data = inputs.make_mixture(n, d, C, 0.5, 33)
    sim = B.Simulation(to_device(data), P=4, K=2, variant=variant, delay_kind="exp", mu=1.0, eta=0.02, m=8, seed=1, n_replicas=R)
    X4 = quantise(data["X"].astype(np.float64))[0]
    for steps in (0, 25):
        if steps:
            sim.run(steps)
        got, exact, w = sim.eval_loss(mxfp4=True), sim.eval_loss(), sim.params()
        assert np.array_equal(got, sim.eval_loss(mxfp4=True))
        for r in (0, R // 2, R - 1):
            W = w[r].reshape(C, d).astype(np.float64)
            W4 = quantise(W)[0]
            z, size, y = X4 @ W4.T, np.abs(X4) @ np.abs(W4).T, data["y"]
            if model == "lsq":
                e = z[:, 0] - y
                want, slope, terms = 0.5 * e * e, np.abs(e)[:, None], 0.5 * e * e
            elif model == "logistic":
                v = z[:, 0]
                want, slope, terms = np.logaddexp(0, v) - y * v, np.ones((n, 1)), 1 + np.abs(v)
            else:
                top = z.max(1)
                want = top + np.log(np.exp(z - top[:, None]).sum(1)) - z[np.arange(n), y]
                slope, terms = np.ones((n, C)), 1 + np.abs(z).sum(1)
            # the logits' sums (d terms, up to 2^-23 of a step each), passed on by the loss's slope, and a few fp32 roundings of its terms
            tol = d * 2.0 ** -23 * (slope * size).sum(1).mean() + 2.0 ** -20 * terms.mean()
            assert abs(got[r] - want.mean()) <= tol, (model, steps, r, got[r], want.mean(), tol)
        if steps:
            assert not np.array_equal(got, exact)           # four bits are seen in the risk
    sim.close()


def test_risk_in_mxfp4_spans_several_products(B):
    """More rows than one product takes (65536): the segments join."""
    n, d = 140001, 8
    data = inputs.make_lsq(n, d, 0.1, 40)
    sim = B.Simulation(to_device(data), P=2, K=1, variant="ksync", delay_kind="exp", mu=1.0, eta=0.1, m=4, seed=1, n_replicas=2)
    sim.run(10)
    got, w = sim.eval_loss(mxfp4=True), sim.params()
    X4 = quantise(data["X"].astype(np.float64))[0]
    for r in range(2):
        W4 = quantise(w[r][None].astype(np.float64))[0]
        e = (X4 @ W4.T)[:, 0] - data["y"]
        want = (0.5 * e * e).mean()
        assert abs(got[r] - want) <= 1e-5 * want
    sim.close()


def test_risk_in_mxfp4_is_refused_for_other_models(B):
    data = inputs.make_mixture(300, 128, 3, 0.5, 36, "mlp2", 64)
    for dat, m in ((None, 1), (to_device(data), 128)):
        sim = B.Simulation(dat, P=2, K=1, variant="ksync", delay_kind="exp", mu=1.0, eta=0.1, m=m, seed=0, n_replicas=1)
        with pytest.raises(B.SimError) as e:
            sim.eval_loss(mxfp4=True)
        assert e.value.status == 1
        sim.close()
