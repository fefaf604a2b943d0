"""Plain 64-bit forms of a worker's operators, written from their formulas (numpy).  Test infrastructure."""
import numpy as np
import torch

EPS = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}      # half a step, relative to the value
TINY = {torch.float32: 2.0**-150, torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25}   # half of the smallest step
E4M3 = np.array([i * 2.0**-9 for i in range(8)] + [(8 + i) * 2.0 ** (e - 10) for e in range(1, 16) for i in range(8)][:-1])


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def act(name, z):
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "relu":
            return np.where(np.isnan(z), z, np.maximum(z, 0.0))
        if name == "gelu":
            return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z**3)))
        if name == "silu":
            return z / (1 + np.exp(-z))
    return z


def slope(name, z):
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "relu":
            return np.where(np.isnan(z), z, (z > 0) * 1.0)
        if name == "gelu":
            c = np.sqrt(2 / np.pi)
            t = np.tanh(c * (z + 0.044715 * z**3))
            return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
        if name == "silu":
            q = 1 / (1 + np.exp(-z))
            return q * (1 + z * (1 - q))
    return np.where(np.isnan(z), z, 1.0)


def keep(x):
    """[rows, cols] -> (values, exponents [rows, blocks], codes' values in units of the scale, padded); blocks with infinities or NaN: NaN, exponent 128."""
    rows, cols = x.shape
    b = np.pad(x, ((0, 0), (0, -cols % 32))).reshape(rows, -1, 32)
    lost = ~np.isfinite(b).all(-1)
    b = np.where(lost[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    k = np.full(top.shape, -127.0)
    live = top > 0
    k[live] = np.ceil(np.log2(top[live] / 448.0))
    k = np.where(live & (448.0 * np.exp2(k) < top), k + 1, k)
    k = np.where(live & (448.0 * np.exp2(k - 1) >= top), k - 1, k)
    k = np.maximum(k, -127.0)
    a = np.abs(b) / np.exp2(k)[..., None]
    hi = np.minimum(np.searchsorted(E4M3, a), len(E4M3) - 1)
    lo = np.maximum(hi - 1, 0)
    down, up = a - E4M3[lo], E4M3[hi] - a
    q = np.copysign(E4M3[np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)], b)
    v = np.where(lost[..., None], np.nan, q * np.exp2(k)[..., None]).reshape(rows, -1)[:, :cols]
    return v, np.where(lost, 128.0, k), q


def values(c):
    """(values [rows, cols], exponents) of a Checkpoint, from its bytes; checks the zero tail."""
    blocks = -(-c.cols // 32)
    codes = c.codes.cpu().view(torch.float8_e4m3fn).to(torch.float64).numpy().reshape(c.rows, blocks, 32)
    k = c.scales.cpu().numpy().astype(np.float64).reshape(c.rows, blocks) - 127
    tail = codes.reshape(c.rows, -1)[:, c.cols:]
    assert not (tail[~np.isnan(tail)] != 0).any(), "the tail of a row must be zero"
    v = np.where((k == 128)[..., None], np.nan, codes * np.exp2(np.minimum(k, 127))[..., None])
    return v.reshape(c.rows, -1)[:, : c.cols], k


def in_range(want, dt):
    """Values that a rounding to dt takes beyond its largest number are infinite: from its last step on."""
    top = float(torch.finfo(dt).max) * (1 + EPS[dt])
    return np.where(np.abs(want) >= top, np.copysign(np.inf, want), want)


def close(got, want, tol, what=""):
    got = f64(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad_nan = np.isnan(got) != np.isnan(want)
    assert not bad_nan.any(), "%s: NaN at %s" % (what, np.argwhere(bad_nan)[:3].tolist())
    with np.errstate(invalid="ignore"):
        off = np.where(np.isnan(want) | (got == want), 0.0, np.abs(got - want) - tol)
    assert (off <= 0).all(), "%s: %d off, first at %s, worst by %g over its tolerance" % (what, (off > 0).sum(), np.argwhere(off > 0)[0].tolist(), off.max())
