"""Gradients of log probabilities at the ends of what a call takes, against 64 bits: masks beside large derivatives and low temperatures.

Tolerances, relative to a probability where nothing else is said.  In powers of two a logit is d = c x - m, c rounded once (2^-24 of it), m exact: what
is common to a row's logits cancels, so a logit's numerator is off by e = 2^-24 (2 |log2 p| + 40) (c and one rounding of d, |d| <= |log2 p| + log2 s, log2 s <= 33
with m up to 16 below the largest) and by the power's own 2^-22.  A sum adds n = 1 + vocab / 128 terms one by one and then a tree of less than 32 levels, and
is moved to another m a few times (2^-20 in all): S = (n + 32) 2^-24 + 2^-20 + the mean of e.  So a probability is off by P = e + S + 2^-21, its logarithm by as much,
and the entropy, logarithms of at most L = 2 log2(vocab) + 10 so weighed, by 2 R (L + 2), R = S + 40 2^-24.  A gradient is (exp2(d) (a d + b) + g) / T, its own
rounding 2^-22 of |a| (|d| + 33) + |b|; then half a step of its type.  A power under 2^-126 may be taken as zero: p is off by 2^-125 at most (s >= 1/2)."""
import numpy as np
import pytest
import torch

from worker_ref import EPS, TINY, close, f64

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def rows_of(x, T):
    """log p, p, entropy of finite or masked (-inf) logits as they are stored; the mean of e."""
    l = x / T
    top = l.max(1, keepdims=True)
    lp = (l - top) - np.log(np.exp(l - top).sum(1, keepdims=True))
    p = np.exp(lp)
    lp = np.where(p > 0, lp, 0.0)
    return lp, p, -(p * lp).sum(1)


def expect(x, t, T, g, h):
    """The gradient and its tolerance."""
    lp, p, H = rows_of(x, T)
    rows, vocab = x.shape
    e = 2.0**-24 * (2 * np.abs(lp) / np.log(2) + 40)
    S = ((33 + vocab / 128) * 2.0**-24 + 2.0**-20 + (p * e).sum(1))[:, None]
    P, L, R = e + S + 2.0**-21, 2 * np.log2(vocab) + 10, S + 40 * 2.0**-24
    d = -p * g[:, None] - h[:, None] * p * (lp + H[:, None])
    ag, ah, size = np.abs(g)[:, None], np.abs(h)[:, None], np.abs(lp) + H[:, None]
    tol = p * (ag * P + ah * (size * P + P + 2 * R * (L + 2))) + (2.0**-22 * p + 2.0**-125) * (ag + ah * (size + 66 + 33))
    r = np.arange(rows)
    d[r, t] += g
    tol[r, t] += 2.0**-22 * np.abs(g)
    return d / T, tol / T, p


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("vocab", [100, 1031, 5003, 50021])
@pytest.mark.parametrize("T,weight", [(0.001, 1e3), (0.001, 1e6), (0.01, 1e5), (0.1, 1e8), (1.0, 1e9)])
def test_masked_logits_beside_large_derivatives_by_entropy(B, dt, vocab, T, weight):
    """What is masked has probability zero and no gradient, however large its factor would be."""
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    x = (torch.randn(5, vocab, generator=gen, device=DEV) * T).to(dt)          # spread by one once divided by T: many classes count
    x[0, ::3] = float("-inf")
    x[1, vocab // 2:] = torch.finfo(dt).min
    x[2, 1::2] = -60000.0 if dt == torch.float16 else -1.5e30
    x[3] = float("-inf")
    x[3, vocab // 2] = 0.5
    t = torch.tensor([1, 0, 2, vocab // 2, 3], device=DEV)
    g = torch.tensor([1.0, -2.0, 0.5, 1.0, 3.0], device=DEV)
    h = torch.tensor([1.0, -1.0, 1.0, 1.0, 0.5], device=DEV) * weight
    want, tol, p = expect(f64(x), t.cpu().numpy(), T, f64(g), f64(h))
    if dt == torch.float16:                                                     # beyond the type's largest number: infinite
        big = np.abs(want) > 60000.0
        want, tol = np.where(big, 0.0, want), np.where(big, 0.0, tol)
    for got in (B.log_probs(x, t, temperature=T, d_logp=g, d_entropy=h).dlogits, B.log_probs_backward(x, t, g, h, temperature=T)):
        d = f64(got)
        assert not np.isnan(d).any() and (d[p == 0] == 0).all()
        if dt == torch.float16:
            d = np.where(big, 0.0, d)
        close(d, want, tol + (EPS[dt] + 2.0**-22) * np.abs(want) + TINY[dt], "dlogits")


@pytest.mark.parametrize("vocab,rows", [(10, 6), (700, 6), (3001, 6), (20011, 4), (50021, 3), (9001, 300)])
@pytest.mark.parametrize("dt,off,spread,T", [(torch.float32, 1e4, 2.5, 1.0), (torch.float32, -1e4, 2.5, 1.0), (torch.float32, 1e6, 2.5, 1.0), (torch.float32, 1e8, 25.0, 1.0), (torch.float32, 300.0, 0.02, 0.01),
                                             (torch.float32, 1e6, 0.1, 0.01), (torch.float16, 6e4, 32.0, 1.0), (torch.float16, 6e4, 32.0, 50.0), (torch.float16, 6e4, 32.0, 0.001), (torch.bfloat16, 1e6, 8000.0, 1000.0),
                                             (torch.bfloat16, 3e4, 100.0, 1.0)])
def test_rows_far_from_zero(B, dt, off, spread, T, vocab, rows):
    """An offset that all logits of a row share changes nothing but lse, and takes no digits from probabilities and gradients."""
    gen = torch.Generator(device=DEV).manual_seed(vocab + rows)
    x = (torch.randn(rows, vocab, generator=gen, device=DEV, dtype=torch.float64) * spread + off).to(dt)
    t = torch.randint(0, vocab, (rows,), generator=gen, device=DEV)
    t[0] = x[0].argmax()
    g, h = torch.randn(rows, generator=gen, device=DEV), torch.randn(rows, generator=gen, device=DEV)
    X, tok = f64(x), t.cpu().numpy()
    lp, p, H = rows_of(X, T)
    lp_t = (X / T - (X / T).max(1, keepdims=True))[np.arange(rows), tok] - np.log(np.exp(X / T - (X / T).max(1, keepdims=True)).sum(1))
    S = (33 + vocab / 128) * 2.0**-24 + 2.0**-20 + 80 * 2.0**-24
    for gg, hh in ((g, h), (g, torch.zeros_like(h)), (torch.zeros_like(g), h)):
        got = B.log_probs(x, t, temperature=T, d_logp=gg, d_entropy=hh)
        want, tol, _ = expect(X, tok, T, f64(gg), f64(hh))
        close(got.dlogits, want, tol + (EPS[dt] + 2.0**-22) * np.abs(want) + TINY[dt], "dlogits")
        if dt == torch.float32:                      # a row's gradient sums to nothing
            assert (np.abs(f64(got.dlogits).sum(1)) <= tol.sum(1) + 2.0**-23 * np.abs(want).sum(1)).all()
    close(got.logp, lp_t, S + 2.0**-22 * np.abs(lp_t), "logp")
    close(got.entropy, H, 2 * S * (2 * np.log2(vocab) + 12), "entropy")
    close(got.lse, (X / T).max(1) + np.log(np.exp(X / T - (X / T).max(1, keepdims=True)).sum(1)), S + 2.0**-22 * np.abs(X / T).max(1) + 2.0**-22 * 40, "lse")


@pytest.mark.parametrize("rows,vocab", [(4, 12), (4, 100), (4, 900), (4, 3001), (3, 20011), (300, 9001)])
@pytest.mark.parametrize("middle,T", [(2e8, 1.0), (-1e9, 1.0), (1e8, 0.1), (-3e6, 0.01), (1.8606e8, 1.0), (-1.8606e8, 1.0), (7e12, 1000.0), (2e37, 1.0), (-2e38, 1.0)])
@pytest.mark.parametrize("order", ["mixed", "rising", "falling"])
def test_logits_a_few_steps_apart_beyond_2_to_the_28(B, rows, vocab, middle, T, order):
    """fp32 logits around masks like -1e9: neighbours are many nats apart, and still told apart.  1.8606e8 is where references begin to be logits."""
    gen = torch.Generator().manual_seed(vocab)
    step = np.spacing(np.float32(abs(middle)))
    k = torch.randint(-9, 10, (rows, vocab), generator=gen).double()
    k = k if order == "mixed" else k.sort(1, descending=order == "falling")[0]
    x = (middle + float(step) * k).float().cuda()
    x[1, : vocab // 2] = float("-inf")
    X, t = f64(x), torch.randint(vocab // 2, vocab, (rows,), generator=gen).cuda()
    t[0] = x[0].argmax()
    g, h = torch.randn(rows, generator=gen).cuda(), torch.randn(rows, generator=gen).cuda()
    tok = t.cpu().numpy()
    top = min(4, vocab)
    got = B.log_probs(x, t, temperature=T, top=top, d_logp=g, d_entropy=h)
    with np.errstate(invalid="ignore"):
        lp, p, H = rows_of(X, T)
        want, tol, _ = expect(X, tok, T, f64(g), f64(h))
    low = (X / T - (X / T).max(1, keepdims=True)) - np.log(p.max(1, keepdims=True) ** -1)
    S = (33 + vocab / 128) * 2.0**-24 + 2.0**-20 + 80 * 2.0**-24
    close(got.dlogits, want, tol + 2.0**-22 * np.abs(want) + TINY[torch.float32], "dlogits")
    lp_t = low[np.arange(rows), tok]
    close(got.logp, lp_t, S + 2.0**-21 * np.abs(lp_t), "logp")
    close(got.entropy, H, 2 * S * (2 * np.log2(vocab) + 12), "entropy")
    close(got.lse, (X / T).max(1) - np.log(p.max(1)), S + 2.0**-21 * np.abs(X / T).max(1, where=np.isfinite(X), initial=0), "lse")
    ids = np.argsort(-X, axis=1, kind="stable")[:, :top]
    assert np.array_equal(got.top_ids.cpu().numpy(), ids)
    at = np.take_along_axis(low, ids, 1)
    close(got.top_logp, at, S + 2.0**-21 * np.abs(at), "top_logp")


@pytest.mark.parametrize("vocab", [100, 900, 3001, 20011])
def test_some_logits_beyond_2_to_the_28(B, vocab):
    """A mask added in fp32 leaves numbers around -1e9 beside the ones that count, wherever they stand and whichever come first."""
    gen = torch.Generator().manual_seed(vocab)
    x = torch.randn(6, vocab, generator=gen)
    x[0, ::2] -= 1e9
    x[1, : vocab - 1] -= 1e9
    x[2, 1:] -= 1e9
    x[3] = x[3] * 100 - 1e9
    x[4, vocab // 2:] += 1e9
    x[5, vocab // 3] = 3e8
    x = x.cuda()
    t = x.argmax(1)
    g, h = torch.randn(6, generator=gen).cuda(), torch.randn(6, generator=gen).cuda()
    X, tok = f64(x), t.cpu().numpy()
    got = B.log_probs(x, t, d_logp=g, d_entropy=h)
    want, tol, p = expect(X, tok, 1.0, f64(g), f64(h))
    close(got.dlogits, want, tol + 2.0**-22 * np.abs(want) + TINY[torch.float32], "dlogits")
    S = (33 + vocab / 128) * 2.0**-24 + 2.0**-20 + 80 * 2.0**-24
    close(got.logp, np.log(p.max(1)), S + 2.0**-21 * np.abs(np.log(p.max(1))), "logp")
    close(got.entropy, rows_of(X, 1.0)[2], 2 * S * (2 * np.log2(vocab) + 12), "entropy")


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [12, 100, 900, 3001, 20011])
def test_logits_beyond_the_range_once_divided(B, dt, vocab):
    """2e38 / 0.1 counts as infinite: the row is NaN; -2e38 / 0.1 as -inf: no probability, and a row of nothing else has no entropy and no gradient."""
    x = torch.zeros(4, vocab, dtype=dt, device=DEV)
    x[0, vocab // 2] = 2e38
    x[1] = 2e38
    x[2] = -2e38
    x[3, 1:] = -2e38
    t = torch.tensor([vocab // 2, 0, 1, 0], device=DEV)
    one = torch.ones(4, device=DEV)
    got = B.log_probs(x, t, temperature=0.1, d_logp=one, d_entropy=one)
    assert all(torch.isnan(r[:2]).all() for r in (got.logp, got.entropy, got.lse, got.dlogits))
    assert got.logp[2] == got.lse[2] == float("-inf") and got.entropy[2] == 0 and got.logp[3] == 0 and got.entropy[3] == 0 and got.lse[3] == 0
    assert (got.dlogits[2:] == 0).all()
