"""Cases of the operators that a worker of a large model runs between fetching parameters and pushing gradients: layers (matrix
products with bias, activation and residual), activations kept in 8 bits until the backward pass, and log probabilities of
given tokens with entropy, the likeliest alternatives and gradients.

Definitions shared by both forms:
  * activations: relu; gelu(z) = z / 2 (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))); silu(z) = z / (1 + exp(-z)).
  * a checkpoint: blocks of 32 along a row, scale 2^k with the smallest k >= -127 for which no magnitude of the block exceeds
    448 * 2^k, elements in E4M3 (units of the scale), nearest even; rows of codes padded with zeros to whole blocks.
  * what an operator returns in a 16-bit type is rounded to it, also where the next operator of the same pass takes it.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}


# ---- cases ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # serving: one token through a layer with its skip connection; the weights' way from memory
        {"name": "linear_one_token", "op": "linear", "M": 1, "K": 4096, "N": 12288, "type": "bf16", "act": "none", "bias": True, "res": True},
        # serving: a handful of sequences, fp16, odd widths as a pruned model has them
        {"name": "linear_37_tokens_odd", "op": "linear", "M": 37, "K": 2051, "N": 5003, "type": "f16", "act": "silu", "bias": True, "res": False},
        # a relu MLP's hidden layer of 512 units for the samples of one update (16 minibatches of 128)
        {"name": "linear_hidden_layer", "op": "linear", "M": 2048, "K": 1024, "N": 512, "type": "bf16", "act": "relu", "bias": True, "res": False},
        # serving: a prompt through a large layer
        {"name": "linear_prompt", "op": "linear", "M": 4096, "K": 8192, "N": 8192, "type": "bf16", "act": "gelu", "bias": True, "res": True},
        # a worker's step through a feed-forward block, ragged number of tokens, odd widths: output and all gradients
        {"name": "block_train_ragged", "op": "block", "T": 1531, "d": 1001, "f": 2731, "act": "silu"},
        # the same at the width of a large model, the largest case
        {"name": "block_train_large", "op": "block", "T": 8192, "d": 4096, "f": 11264, "act": "gelu"},
        # what one layer keeps of a single sequence of 77 tokens: latency
        {"name": "checkpoint_77_tokens", "op": "keep", "rows": 77, "cols": 768, "type": "f16", "act": "relu"},
        # what one layer keeps of a large batch, read back and used
        {"name": "checkpoint_batch", "op": "keep", "rows": 16384, "cols": 11264, "type": "bf16", "act": "gelu"},
        # ten classes of the simulated softmax workers, all samples of the data set, loss gradient included
        {"name": "logprobs_ten_classes", "op": "logp", "rows": 65536, "vocab": 10, "type": "f32", "top": 3, "temp": 1.0, "grad": True},
        # sampling: a few sequences, a large vocabulary of odd length, temperature, twenty alternatives
        {"name": "logprobs_decode", "op": "logp", "rows": 8, "vocab": 100277, "type": "bf16", "top": 20, "temp": 0.7, "grad": False},
        # scoring a batch of sequences with alternatives
        {"name": "logprobs_score", "op": "logp", "rows": 4096, "vocab": 131072, "type": "bf16", "top": 8, "temp": 1.0, "grad": False},
        # training: loss gradient with an entropy bonus, no alternatives
        {"name": "logprobs_train", "op": "logp", "rows": 8192, "vocab": 50021, "type": "bf16", "top": 0, "temp": 1.0, "grad": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "block", "keep", "logp", "logp"])
    act = rng.choice(["relu", "gelu", "silu"])
    if kind == "linear":
        return {"op": "linear", "M": _log(rng, 1, 4096), "K": _log(rng, 24, 8192), "N": _log(rng, 16, 8192), "type": rng.choice(["bf16", "f16"]),
                "act": rng.choice(["none", act]), "bias": rng.random() < 0.7, "res": rng.random() < 0.5}
    if kind == "block":
        return {"op": "block", "T": _log(rng, 1, 6000), "d": _log(rng, 16, 3000), "f": _log(rng, 32, 8000), "act": act}
    if kind == "keep":
        return {"op": "keep", "rows": _log(rng, 1, 12000), "cols": _log(rng, 5, 11000), "type": rng.choice(["bf16", "f16", "f32"]), "act": act}
    vocab = _log(rng, 2, 260000)
    return {"op": "logp", "rows": _log(rng, 1, min(65536, (1 << 28) // vocab)), "vocab": vocab, "type": rng.choice(["bf16", "f16", "f32"]),
            "top": rng.choice([0, 1, min(5, vocab), min(20, vocab), min(32, vocab)]), "temp": rng.choice([1.0, 0.6, 1.3]), "grad": rng.random() < 0.5}


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device=DEV).mul_(scale).to(dtype)

    s = {"case": case}
    if case["op"] == "linear":
        M, K, N, dt = case["M"], case["K"], case["N"], TYPES[case["type"]]
        s["x"], s["w"] = normal(M, K, dtype=dt), normal(N, K, scale=K**-0.5, dtype=dt)
        s["b"] = normal(N, scale=0.3, dtype=dt) if case["bias"] else None
        s["r"] = normal(M, N, dtype=dt) if case["res"] else None
    elif case["op"] == "block":
        T, d, f = case["T"], case["d"], case["f"]
        s["x"], s["dy"] = normal(T, d, dtype=torch.bfloat16), normal(T, d, scale=0.01, dtype=torch.bfloat16)
        s["w1"], s["w2"] = normal(f, d, scale=d**-0.5, dtype=torch.bfloat16), normal(d, f, scale=f**-0.5, dtype=torch.bfloat16)
        s["b1"], s["b2"] = normal(f, scale=0.3), normal(d, scale=0.3)
    elif case["op"] == "keep":
        rows, cols, dt = case["rows"], case["cols"], TYPES[case["type"]]
        s["x"] = (normal(rows, cols) * torch.exp(0.7 * normal(rows, 1))).to(dt)
        s["dy"] = normal(rows, cols, scale=0.01, dtype=dt)
    else:
        rows, vocab = case["rows"], case["vocab"]
        x = normal(rows, vocab, scale=2.5)
        if vocab > 1000:       # a vocabulary padded to a round length, and tokens that a row may not take, are masked
            x[:, vocab - vocab // 997:] = -math.inf
            x[::3, 7: vocab // 11] = -math.inf
        tokens = torch.randint(vocab // 11 if vocab > 1000 else 0, vocab - vocab // 997 if vocab > 1000 else vocab, (rows,), generator=gen, device=DEV)
        x[torch.arange(0, rows, 2, device=DEV), tokens[::2]] += 9.0     # a trained model is sure of many of them
        s["tokens"] = torch.where(torch.rand(rows, generator=gen, device=DEV) < 0.1, torch.full_like(tokens, -100), tokens)     # padding of the batch
        s["x"] = x.to(TYPES[case["type"]])
        if case["grad"]:
            s["d_logp"], s["d_ent"] = normal(rows, scale=1.0 / rows), normal(rows, scale=0.01 / rows)
    return s


# ---- plain forms, 32 bits ----------------------------------------------------------------------------------------------------
def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    if name == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _pow2(k):
    """2^k in 32 bits, -127 <= k <= 127, from its bits (2^-127 is subnormal)."""
    return torch.where(k > -127, (k + 127) << 23, torch.full_like(k, 1 << 22)).view(torch.float32)


def _keep(x):
    """(E4M3 elements in units of the scale, exponents) of the rows of x, in blocks of 32."""
    b = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % 32)).unflatten(1, (-1, 32))
    frac, e = torch.frexp(b.abs().amax(-1))
    k = torch.where(frac > 0, e - 9 + (frac > 0.875).to(e.dtype), torch.full_like(e, -127)).clamp(min=-127)
    a = b * _pow2(-k)[..., None]
    step = _pow2((torch.frexp(a)[1] - 1).clamp(min=-6) - 3)
    return torch.round(a / step) * step, k


def _kept(q, k, cols):
    return (q * _pow2(k)[..., None]).flatten(1)[:, :cols]


def _block_plain(s):
    act = s["case"]["act"]
    x, dy, w1, w2 = (s[n].float() for n in ("x", "dy", "w1", "w2"))
    T, d, f = s["case"]["T"], s["case"]["d"], s["case"]["f"]
    kept_x = _kept(*_keep(x), d)
    z = x @ w1.t() + s["b1"]
    h = _act(act, z).to(torch.bfloat16).float()
    kept_z = _kept(*_keep(z), f)
    y = h @ w2.t() + s["b2"] + x
    h = _act(act, kept_z).to(torch.bfloat16).float()
    dz = ((dy @ w2) * _slope(act, kept_z)).to(torch.bfloat16).float()
    out = {"y": y, "dx": dz @ w1 + dy, "dw1": dz.t() @ kept_x, "db1": dz.sum(0), "dw2": dy.t() @ h, "db2": dy.sum(0)}
    return {n: t.to(torch.bfloat16) for n, t in out.items()}


def _logp_plain(s):
    case, rows, vocab = s["case"], s["case"]["rows"], s["case"]["vocab"]
    x = s["x"].float()
    l = x / case["temp"]
    lse = torch.logsumexp(l, 1)
    logp = l - lse[:, None]
    p = torch.exp(logp)
    ent = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    live = s["tokens"] >= 0
    at = s["tokens"].clamp(min=0)[:, None]
    out = {"logp": torch.where(live, logp.gather(1, at)[:, 0], torch.zeros_like(lse)), "entropy": ent, "lse": lse}
    if case["top"]:
        bits = s["x"].float().view(torch.int32).long()                      # order of the numbers, the lower index first among equals
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * 2**20 + (vocab - 1 - torch.arange(vocab, device=DEV))
        ids = torch.topk(key, case["top"], dim=1).indices
        out["top_ids"], out["top_logp"] = ids.int(), logp.gather(1, ids)
    if case["grad"]:
        g = torch.where(live, s["d_logp"], torch.zeros_like(lse))[:, None]
        grad = -p * (g + s["d_ent"][:, None] * torch.where(p > 0, logp + ent[:, None], torch.zeros_like(p)))
        grad.scatter_add_(1, at, g)
        out["dlogits"] = (grad / case["temp"]).to(s["x"].dtype)
    return out


# ---- one pass ----------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        from paper_2003_10579_b200 import binding as B
    if case["op"] == "linear":
        if own:
            return B.linear(s["x"], s["w"], s["b"], act=case["act"], residual=s["r"])
        y = s["x"].float() @ s["w"].float().t()
        if s["b"] is not None:
            y = y + s["b"].float()
        y = _act(case["act"], y)
        if s["r"] is not None:
            y = y + s["r"].float()
        return y.to(s["x"].dtype)
    if case["op"] == "block":
        if not own:
            return _block_plain(s)
        act, bf16 = case["act"], torch.bfloat16
        x = B.checkpoint(s["x"])
        h, z = B.linear(s["x"], s["w1"], s["b1"], act=act, keep=True)
        y = B.linear(h, s["w2"], s["b2"], residual=s["x"])
        del h                                    # between the passes only the 8-bit forms stay
        dz, dw2, db2 = B.linear_backward(s["dy"], z, s["w2"], x_act=act, dtype=bf16)
        dx, dw1, db1 = B.linear_backward(dz, x, s["w1"], residual=s["dy"], dtype=bf16)
        return {"y": y, "dx": dx, "dw1": dw1, "db1": db1, "dw2": dw2, "db2": db2}
    if case["op"] == "keep":
        act, dt = case["act"], TYPES[case["type"]]
        if own:
            q = B.checkpoint(s["x"])
            h = B.checkpoint_read(q, dt, act=act)
            dz, db = B.act_backward(s["dy"], q, act)
            return {"codes": q.codes.view(torch.float8_e4m3fn), "scales": q.scales.view(torch.float8_e8m0fnu), "h": h, "dz": dz, "db": db}
        q, k = _keep(s["x"])
        z = _kept(q, k, case["cols"])
        dz = s["dy"].float() * _slope(act, z)
        return {"codes": q.flatten().to(torch.float8_e4m3fn), "scales": (k + 127).to(torch.uint8).flatten().view(torch.float8_e8m0fnu), "h": _act(act, z).to(dt),
                "dz": dz.to(dt), "db": dz.sum(0)}
    if not own:
        return _logp_plain(s)
    r = B.log_probs(s["x"], s["tokens"], top=case["top"], temperature=case["temp"], d_logp=s.get("d_logp"), d_entropy=s.get("d_ent"))
    out = {"logp": r.logp, "entropy": r.entropy, "lse": r.lse}
    if case["top"]:
        out["top_ids"], out["top_logp"] = r.top_ids, r.top_logp
    if case["grad"]:
        out["dlogits"] = r.dlogits
    return out


# ---- work and exact values ---------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": 2.0 * (M * K + N * K + M * N * (2 if case["res"] else 1)), "flops": 2.0 * M * N * K}
    if case["op"] == "block":
        T, d, f = case["T"], case["d"], case["f"]
        return {"bytes": 2.0 * (4 * T * d + 4 * d * f) + 6.0 * (d + f), "flops": 12.0 * T * d * f}
    if case["op"] == "keep":
        n, b = case["rows"] * case["cols"], SIZE[case["type"]]
        return {"bytes": n * (2 * b + 33.0 / 32 + 2 * b) + 4.0 * case["cols"], "flops": 40.0 * n}
    n, b = case["rows"] * case["vocab"], SIZE[case["type"]]
    return {"bytes": n * b * (2 if case["grad"] else 1) + case["rows"] * (16.0 + 8.0 * case["top"]), "flops": n * (14.0 if case["grad"] else 6.0)}


_GRID = [i * 2.0**-9 for i in range(8)] + [(8 + i) * 2.0 ** (e - 10) for e in range(1, 16) for i in range(8)][:-1]


def _keep64(x):
    """Blocks of 32 against the list of E4M3's values, in 64 bits: the nearer neighbour, at the middle the even place of the list."""
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    q = torch.empty(x.shape[0], -(-x.shape[1] // 32), 32, dtype=torch.float64, device=x.device)
    k = torch.empty(q.shape[:2], dtype=torch.float64, device=x.device)
    slab = max(1, 30000000 // x.shape[1])
    for at in range(0, x.shape[0], slab):
        b = torch.nn.functional.pad(x[at: at + slab].double(), (0, -x.shape[1] % 32)).unflatten(1, (-1, 32))
        top = b.abs().amax(-1)
        e = torch.ceil(torch.log2(top / 448))
        e = torch.where(448 * torch.exp2(e) < top, e + 1, e)
        e = torch.where(448 * torch.exp2(e - 1) >= top, e - 1, e).clamp(min=-127)
        a = b.abs() / torch.exp2(e)[..., None]
        hi = torch.searchsorted(grid, a).clamp(max=len(_GRID) - 1)
        lo = (hi - 1).clamp(min=0)
        down, up = a - grid[lo], grid[hi] - a
        pick = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
        q[at: at + slab], k[at: at + slab] = torch.copysign(grid[pick], b), e
    return q, k


def _act64(name, z):
    """(activation, derivative) by the logistic function: gelu in its tanh form is z times that of twice the tanh's argument."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), torch.sign(z).clamp(min=0)
    if name == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    c = 2 * math.sqrt(2 / math.pi)
    q = torch.sigmoid(c * (z + 0.044715 * z**3))
    return z * q, q + z * q * (1 - q) * c * (1 + 0.134145 * z**2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        z = s["x"].double() @ s["w"].double().t()
        if s["b"] is not None:
            z += s["b"].double()
        z = _act64(case["act"], z)[0]
        return z if s["r"] is None else z + s["r"].double()
    if case["op"] == "block":
        x, dy, w1, w2 = (s[n].double() for n in ("x", "dy", "w1", "w2"))
        z = x @ w1.t() + s["b1"].double()
        h = _act64(case["act"], z)[0].to(torch.bfloat16).double()
        y = h @ w2.t() + s["b2"].double() + x
        q, k = _keep64(z)
        h, slope = _act64(case["act"], (q * torch.exp2(k)[..., None]).flatten(1)[:, : case["f"]])
        h = h.to(torch.bfloat16).double()
        dz = ((dy @ w2) * slope).to(torch.bfloat16).double()
        q, k = _keep64(x)
        x = (q * torch.exp2(k)[..., None]).flatten(1)[:, : case["d"]]
        return {"y": y, "dx": dz @ w1 + dy, "dw1": dz.t() @ x, "db1": dz.sum(0), "dw2": dy.t() @ h, "db2": dy.sum(0)}
    if case["op"] == "keep":
        q, k = _keep64(s["x"])
        n, cols = case["rows"], case["cols"]
        h, dz = torch.empty(n, cols, dtype=torch.float64, device=DEV), torch.empty(n, cols, dtype=torch.float64, device=DEV)
        for at in range(0, n, 2048):
            rows = slice(at, at + 2048)
            h[rows], slope = _act64(case["act"], (q[rows] * torch.exp2(k[rows])[..., None]).flatten(1)[:, :cols])
            dz[rows] = slope * s["dy"][rows].double()
        return {"codes": q.flatten(), "scales": torch.exp2(k).flatten(), "h": h, "dz": dz, "db": dz.sum(0)}
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    out = {n: torch.zeros(rows, dtype=torch.float64, device=DEV) for n in ("logp", "entropy", "lse")}
    if top:
        out["top_ids"], out["top_logp"] = None, torch.empty(rows, top, dtype=torch.float64, device=DEV)
    if case["grad"]:
        out["dlogits"] = torch.empty(rows, vocab, dtype=torch.float64, device=DEV)
    slab = max(1, 60000000 // vocab)
    for at in range(0, rows, slab):
        r = slice(at, min(rows, at + slab))
        x = s["x"][r].double() / case["temp"]
        most = x.amax(1, keepdim=True)
        x = x - most
        e = torch.exp(x)
        total = e.sum(1, keepdim=True)
        logp, p = x - torch.log(total), e / total
        ent = -torch.special.xlogy(p, p).sum(1)
        live, at_token = s["tokens"][r] >= 0, s["tokens"][r].clamp(min=0)[:, None]
        out["logp"][r] = logp.gather(1, at_token)[:, 0].masked_fill(~live, 0.0)
        out["entropy"][r], out["lse"][r] = ent, (most + torch.log(total))[:, 0]
        if top:
            out["top_logp"][r] = torch.topk(logp, top, dim=1).values
        if case["grad"]:
            g = s["d_logp"][r].double().masked_fill(~live, 0.0)[:, None]
            d = -g * p - s["d_ent"][r].double()[:, None] * (torch.special.xlogy(p, p) + p * ent[:, None])
            out["dlogits"][r] = d.scatter_add(1, at_token, g) / case["temp"]
    return out
