"""Log probabilities, entropies, alternatives and gradients against 64 bits.

Tolerances.  l = x / T is taken as x times a rounded constant, minus a whole number, in one rounding: off by D = 2^-22 max|l| + 2^-22 (finite l).
A power of two adds 2^-22 of itself.  A sum adds up n terms of a thread one by one and then a tree of less than 32 levels: (n + 32) 2^-24,
n = 1 + vocab / 128 at most.  R, the three together, bounds the relative error of every probability's numerator and of the sums, so lse and logp
are off by 2 R plus the roundings of the results (2^-23 of |lse|, |logp|).  The entropy weighs logarithms of at most L = 2 log2(vocab) + 10
(in 2^d, 2^-8.5 <= s) with such probabilities: 2 R (L + 2).  A gradient -p (g + h (log p + H)) is off by p's 4 R of its terms' magnitudes, by
2^-21 of them for its own arithmetic, by p |h| times the absolute errors of log p and of H (2 R and 2 R (L + 2), whatever their size: with
one class both are zero and their errors are not), and by half a step of its type."""
import numpy as np
import pytest
import torch

from worker_ref import EPS, TINY, close, f64, in_range

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_2003_10579_b200 import binding
    return binding


def reference(x, tokens, T, top, g=None, h=None):
    rows, vocab = x.shape
    with np.errstate(all="ignore"):
        l = x / T
        most = l.max(1, keepdims=True)
        e = np.exp(l - np.where(np.isfinite(most), most, 0.0))
        s = e.sum(1, keepdims=True)
        none = (x == -np.inf).all(1)
        lse = np.where(none, -np.inf, (most + np.log(s))[:, 0])
        bad = np.isnan(x).any(1) | (x == np.inf).any(1)
        lse[bad] = np.nan
        lp = np.where(none[:, None], -np.inf, (l - most) - np.log(s))       # not l - lse: beside 1e38 even 64 bits lose log s
        lp[bad] = np.nan
        p = np.where(none[:, None], 0.0, np.exp(lp))
        ent = -np.where(p > 0, p * lp, 0.0).sum(1)
        ent[bad] = np.nan
        r = np.arange(rows)
        logp = np.where(tokens < 0, 0.0, np.where(tokens >= vocab, np.nan, lp[r, np.clip(tokens, 0, vocab - 1)])) if tokens is not None else None
        key = np.where(np.isnan(x), np.inf, x)
        order = np.lexsort((np.broadcast_to(np.arange(vocab), x.shape), -key, ~np.isnan(x)), axis=1) if top else None
        ids = order[:, :top] if top else None
        out = {"lse": lse, "lp": lp, "p": p, "entropy": ent, "logp": logp, "ids": ids, "top": np.take_along_axis(lp, ids, 1) if top else None, "none": none}
        if g is not None or h is not None:
            g = np.zeros(rows) if g is None else np.where(tokens < 0, 0.0, np.where(tokens >= vocab, np.nan, g))
            h = np.zeros(rows) if h is None else h
            size = p * (np.abs(g)[:, None] + np.abs(h)[:, None] * (np.where(p > 0, np.abs(lp), 0.0) + ent[:, None]))
            d = -p * g[:, None] - h[:, None] * np.where(p > 0, p * (lp + ent[:, None]), 0.0 * p)
            if tokens is not None:
                live = (tokens >= 0) & (tokens < vocab)
                d[r[live], tokens[live]] += g[live]
            d[none] = 0.0
            d[bad] = np.nan
            out["d"], out["size"], out["ph"] = d / T, size / T, p * np.abs(h)[:, None] / T
    return out


def check(B, x, tokens=None, T=1.0, top=0, g=None, h=None, out=None, got=None):
    X = f64(x).reshape(-1, x.shape[-1])
    rows, vocab = X.shape
    t = None if tokens is None else tokens.cpu().numpy().astype(np.int64).reshape(-1)
    want = reference(X, t, T, top, None if g is None else f64(g), None if h is None else f64(h))
    again = got is None
    got = got or B.log_probs(x, tokens, top=top, temperature=T, d_logp=g, d_entropy=h, out=out)
    with np.errstate(all="ignore"):
        # logits that count; where the largest is beyond 2^22, only equal ones do in these tests, and equal ones differ by nothing
        size = np.where(np.isfinite(X) & (want["p"] > 0) & (np.abs(X) < 2.0**22), np.abs(X), 0.0).max(1) / T
    R = 2.0**-22 * (size + 1) + 2.0**-22 + (33 + vocab / 128) * 2.0**-24
    L = 2 * np.log2(vocab) + 10
    fin = lambda a: np.where(np.isfinite(a), np.abs(a), 0.0)  # noqa: E731
    close(got.lse, in_range(want["lse"], torch.float32), 2 * R + 2.0**-23 * fin(want["lse"]), "lse")
    close(got.entropy, want["entropy"], 2 * R * (L + 2), "entropy")
    want = {k: in_range(v, torch.float32) if k in ("lse", "logp", "top") and v is not None else v for k, v in want.items()}
    if tokens is not None:
        close(got.logp, want["logp"], 2 * R + 2.0**-23 * fin(want["logp"]), "logp")
    if top:
        assert np.array_equal(got.top_ids.cpu().numpy(), want["ids"]), "ids"
        close(got.top_logp, want["top"], 2 * R[:, None] + 2.0**-23 * fin(want["top"]), "top")
    if g is not None or h is not None:
        eps = EPS[x.dtype]
        tol = want["size"] * (4 * R + 2.0**-21)[:, None] + want["ph"] * (2 * R + 2 * R * (L + 2))[:, None] + (eps + 2.0**-22) * fin(want["d"]) + TINY[x.dtype]
        if g is not None:
            gg = np.abs(f64(g)) / T
            live = (t >= 0) & (t < vocab)
            tol[np.arange(rows)[live], t[live]] += 2.0**-22 * gg[live]
        close(got.dlogits.reshape(rows, vocab), want["d"], np.nan_to_num(tol) , "dlogits")
    if again and (g is not None or h is not None):
        again = B.log_probs_backward(x, tokens, g, h, temperature=T)
        assert torch.equal(again.view(torch.uint8), got.dlogits.contiguous().view(torch.uint8)), "the backward pass alone"
    return got


def logits(rows, vocab, dt, seed, scale=3.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn(rows, vocab, generator=gen, device=DEV) * scale).to(dt)
    t = torch.randint(-2, vocab, (rows,), generator=gen, device=DEV)
    return x, t, torch.randn(rows, generator=gen, device=DEV), torch.randn(rows, generator=gen, device=DEV)


VOCABS = [1, 2, 10, 16, 17, 100, 128, 129, 1000, 1024, 1025, 2003, 8192, 8193, 20011, 70001]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_over_vocabularies(B, dt, vocab):
    for rows, T, top in ((1, 1.0, 32), (3, 0.7, 1), (37 if vocab < 9000 else 5, 1.5, 5)):
        x, t, g, h = logits(rows, vocab, dt, vocab + rows)
        check(B, x, t, T, min(top, vocab), g, h)
    check(B, x, t.int(), 1.0, 0, g, None)
    check(B, x, None, 1.0, min(3, vocab), None, h)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("vocab,rows", [(40000, 2), (131072, 1), (262147, 3), (50000, 400), (300, 5000)])
def test_few_long_rows_and_many(B, dt, vocab, rows):
    x, t, g, h = logits(rows, vocab, dt, 17)
    if rows > 100:          # compared on a sample of rows: every row has its own block or warp
        pick = torch.tensor([0, 1, rows // 2, rows - 1], device=DEV)
        got = B.log_probs(x, t, top=20, d_logp=g, d_entropy=h)
        rows = type(got)(*(None if r is None else r[pick] for r in got))
        check(B, x[pick], t[pick], 1.0, 20, g[pick], h[pick], got=rows)
    else:
        check(B, x, t, 0.9, 20, g, h)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("vocab", [10, 100, 700, 3001, 20011])
def test_masks(B, dt, vocab):
    """Nothing left, one left, fewer left than alternatives asked for, the type's lowest value as a mask, NaN and infinities."""
    top = min(12, vocab)
    low = torch.finfo(dt).min
    x, _, g, h = logits(12, vocab, dt, 3)
    x[0] = float("-inf")
    x[1] = float("-inf")
    x[1, vocab // 2] = 2.0
    x[2, :] = float("-inf")
    x[2, 1::max(1, vocab // 5)] = 1.0
    x[3] = low
    x[4, : vocab // 2] = low
    x[5] = low
    x[5, vocab - 1] = 1.5
    x[6, vocab // 3] = float("nan")
    x[7, vocab // 4] = float("inf")
    x[8, ::2] = float("-inf")
    x[9] = 0.0
    x[9, 1] = -0.0
    x[10] = 30000.0
    x[11, 3] = float("nan")
    x[11, 0] = float("nan")
    t = torch.tensor([1, vocab // 2, 0, 4, 1, vocab - 1, 0, vocab // 4, 1, 5, 6, vocab + 3], device=DEV)
    check(B, x, t, 1.0, top)
    check(B, x, t, 0.5, top, None, None)
    check(B, x, t, 1.0, top, g, None)
    check(B, x, t, 1.0, top, g, h)


@pytest.mark.parametrize("dt", TYPES)
def test_ties_go_to_the_lowest_index(B, dt):
    for vocab in (40, 900, 5000, 30011):
        x = torch.zeros(4, vocab, device=DEV)
        x[1] = (torch.arange(vocab, device=DEV) // 7 % 5).float()
        x[2] = torch.linspace(8, -8, vocab, device=DEV)
        x[3, vocab // 2:] = 1.0
        check(B, x.to(dt), None, 1.0, 32)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("vocab,pad,off", [(10, 3, 1), (999, 1, 1), (5003, 5, 3), (30011, 8, 0), (30011, 1, 1)])
def test_strides_alignment_and_gradients_in_place(B, dt, vocab, pad, off):
    rows = 5
    x, t, g, h = logits(rows, vocab, dt, 9)
    full = torch.full((rows * (vocab + pad) + 8,), 5.0, dtype=dt, device=DEV)
    v = full[off: off + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    v.copy_(x)
    want = B.log_probs(x, t, top=min(7, vocab), d_logp=g, d_entropy=h)
    check(B, v, t, 1.0, min(7, vocab), g, h)
    frame = torch.full((rows * (vocab + 6) + 9,), 3.0, dtype=dt, device=DEV)
    out = frame[3: 3 + rows * (vocab + 6)].view(rows, vocab + 6)[:, :vocab]
    check(B, v, t, 1.0, 0, g, h, out=out)
    assert (frame[3: 3 + rows * (vocab + 6)].view(rows, vocab + 6)[:, vocab:] == 3.0).all() and (frame[:3] == 3.0).all()
    got = B.log_probs(v, t, top=min(7, vocab), d_logp=g, d_entropy=h, out=v)
    assert torch.equal(got.top_ids, want.top_ids) and got.dlogits is v
    check(B, x, t, 1.0, min(7, vocab), g, h, got=got)
    assert (full[off: off + rows * (vocab + pad)].view(rows, vocab + pad)[:, vocab:] == 5.0).all()


def test_sure_rows_keep_their_digits(B):
    """A logit far above the others: its log probability is minus the others' weight, not the difference of two large numbers."""
    for vocab in (12, 300, 4000, 40000):
        x = torch.zeros(3, vocab, device=DEV)
        x[:, 5] = torch.tensor([25.0, 30.0, 60.0], device=DEV)
        got = B.log_probs(x, torch.full((3,), 5, device=DEV))
        want = -np.log1p((vocab - 1) * np.exp(-np.array([25.0, 30.0, 60.0])))
        # half a step of the sum 2^d + rest around 2^d, d <= 1/2: 2^-23, and log2's own rounding
        assert (np.abs(f64(got.logp) - want) <= 2.0**-21).all()


def test_gradient_against_differences(B):
    x, t, g, h = logits(4, 50, torch.float32, 21)
    for T in (1.0, 0.6):
        d = f64(B.log_probs(x, t, temperature=T, d_logp=g, d_entropy=h).dlogits)
        X, tok = f64(x), t.cpu().numpy()

        def loss(X):
            r = reference(X, tok, T, 0)
            return (np.where(tok < 0, 0.0, f64(g)) * r["logp"]).sum() + (f64(h) * r["entropy"]).sum()

        for i in range(4):
            for j in range(0, 50, 3):
                up, down = X.copy(), X.copy()
                up[i, j] += 1e-5
                down[i, j] -= 1e-5
                assert abs(d[i, j] - (loss(up) - loss(down)) / 2e-5) <= 2e-5


def test_one_row_no_rows_streams_and_graphs(B):
    x, t, g, h = logits(6, 20000, torch.bfloat16, 31)
    want = B.log_probs(x, t, top=9, d_logp=g, d_entropy=h)
    one = B.log_probs(x[2], t[2:3], top=9, d_logp=g[2:3], d_entropy=h[2:3])
    assert torch.equal(one.top_ids[0], want.top_ids[2]) and one.dlogits.shape == (20000,)
    empty = B.log_probs(x[:0], t[:0], top=3, d_logp=g[:0])
    assert empty.logp.shape == (0,) and empty.top_ids.shape == (0, 3) and empty.dlogits.shape == (0, 20000)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = B.log_probs(x, t, top=9, d_logp=g, d_entropy=h, stream=st)
    st.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.log_probs(x, t, top=9, d_logp=g, d_entropy=h)
    y, t2, _, _ = logits(6, 20000, torch.bfloat16, 32)
    x.copy_(y)
    t.copy_(t2)
    want = B.log_probs(x, t, top=9, d_logp=g, d_entropy=h)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_rows_far_apart(B):
    """Offsets beyond 2^31 elements."""
    x = torch.zeros(3, 1 << 30, dtype=torch.bfloat16, device=DEV)
    small, t, g, h = logits(3, 3000, torch.bfloat16, 41)
    x[:, :3000] = small
    for n in (11, 600, 3000):
        check(B, x[:, :n], t.clamp(max=n - 1), 1.0, 4, g, h)
    del x
