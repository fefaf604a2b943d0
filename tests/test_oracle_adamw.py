"""The oracle's AdamW server, pinned to torch.optim.AdamW in 64 bits on the same gradients (P = K = 1: serial minibatch steps)."""
import numpy as np
import torch

from oracle import core, models
from oracle.sim import OracleReplica
from paper_2003_10579_b200 import inputs


def test_oracle_adamw_is_torchs_adamw():
    data = inputs.make_logistic(400, 24, 0.1, 5)
    w0 = np.random.default_rng(0).standard_normal(24).astype(np.float32)
    b1, b2, eps, decay, eta = 0.9, 0.98, 1e-7, 0.1, float(np.float32(0.02))
    o = OracleReplica(model="logistic", X=data["X"], y=data["y"], w0=w0, P=1, K=1, variant="ksync", delay_kind="exp", mu=1.0, eta=eta, m=8, seed=3, replica=0,
                      adamw=(b1, b2, eps, decay))
    p = torch.nn.Parameter(torch.from_numpy(w0.astype(np.float64)))
    opt = torch.optim.AdamW([p], lr=eta, betas=(b1, b2), eps=eps, weight_decay=decay)
    for j in range(30):
        idx = core.minibatch_indices(3, 0, 0, j, 400, 8)
        g = models.loss_and_grad("logistic", p.detach().numpy().astype(np.float32), data["X"][idx], data["y"][idx], 1, 0, True)[1]
        p.grad = torch.from_numpy(np.asarray(g, np.float64))
        opt.step()
        o.run(1)
        # the oracle rounds its parameters to fp32 every update, torch's stay in 64 bits; the gradients differ by as much
        assert np.allclose(o.w, p.detach().numpy(), rtol=0, atol=(j + 1) * 2.0 ** -22)
        with torch.no_grad():
            p.copy_(torch.from_numpy(o.w.astype(np.float64)))


def test_oracle_adamw_averages_the_contributors():
    """K = P on one data row: K equal gradients have the mean of one, so the trajectory is that of K = 1."""
    X, y = np.ones((1, 4), np.float32), np.zeros(1, np.float32)
    kw = dict(model="lsq", X=X, y=y, w0=np.ones(4, np.float32), delay_kind="exp", mu=1.0, eta=0.1, m=2, seed=0, replica=0, adamw=(0.9, 0.999, 1e-8, 0.0))
    a = OracleReplica(P=1, K=1, variant="ksync", **kw).run(5)
    b = OracleReplica(P=3, K=3, variant="ksync", **kw).run(5)
    assert np.allclose(a.w, b.w, rtol=0, atol=5 * 2.0 ** -23)
