"""Cases of the operators a parameter server of language-model size needs beside the simulated one: an AdamW step over many
tensors (states in 32 or in 8 bits, one or several pushed gradients averaged on the way, pushes in MXFP4 included), MXFP4
quantisation and reading back, and products of MXFP4 operands.

Definitions shared by both forms:
  * MXFP4: blocks of 32 along a row; scale 2^k with the smallest k for which no magnitude of the block exceeds 6 * 2^k;
    elements on the grid 0, .5, 1, 1.5, 2, 3, 4, 6 (times the scale).
  * 8-bit states: m and sqrt(v) in E4M3, blocks of 32 with a scale 2^k, k the smallest for which no magnitude exceeds
    448 * 2^k; stochastic rounding: |x| -> step * floor(|x| / step + u), u a multiple of 2^-16 in [0, 1).
  * the 16-bit random numbers of stochastic rounding come from Philox4x32-10 (key = seed), eight per counter.
"""
import math

import torch

own = False

DEV = "cuda"
BETAS, EPS, DECAY, LR, STEP = (0.9, 0.999), 1e-8, 0.01, 1e-4, 1000
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4.0, "bf16": 2.0, "mx": 17.0 / 32.0}


# ---- cases ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the server of the logistic workload (4096 features, 4 pushes an update) stepping with AdamW: latency
        {"name": "adamw32_server_4096", "op": "adamw", "bits": 32, "p": "f32", "g": "f32", "K": 4, "sizes": "4096,1", "shadow": False, "pad": True},
        # norms, biases and small matrices of a model, hundreds of ragged tensors back to back in one buffer (no alignment)
        {"name": "adamw32_many_ragged", "op": "adamw", "bits": 32, "p": "f32", "g": "f32", "K": 1, "sizes": "ragged:400:5000", "shadow": False, "pad": False},
        # one block of a small language model held in bf16 throughout
        {"name": "adamw32_block_bf16", "op": "adamw", "bits": 32, "p": "bf16", "g": "bf16", "K": 1, "sizes": "block:1024:2816:1", "shadow": False, "pad": True},
        # five blocks, fp32 master weights, bf16 gradients, the bf16 copy that the workers fetch written on the way
        {"name": "adamw32_blocks_master", "op": "adamw", "bits": 32, "p": "f32", "g": "bf16", "K": 1, "sizes": "block:2048:5632:5", "shadow": True, "pad": True},
        # 8-bit states, a small model of odd widths
        {"name": "adamw8_ragged_block", "op": "adamw", "bits": 8, "p": "f32", "g": "bf16", "K": 1, "sizes": "block:520:1391:2", "shadow": False, "pad": True},
        # the server averages four MXFP4 pushes and steps
        {"name": "adamw8_four_mx_pushes", "op": "adamw", "bits": 8, "p": "f32", "g": "mx", "K": 4, "sizes": "block:1536:4096:2", "shadow": True, "pad": True},
        # the largest: a server's shard of a large model in one go
        {"name": "adamw8_large_shard", "op": "adamw", "bits": 8, "p": "f32", "g": "bf16", "K": 1, "sizes": "block:4096:11264:1", "shadow": False, "pad": True},
        # a worker's gradient pushed in 4 bits and read back by the server: one flat vector of odd length
        {"name": "mx_push_and_read", "op": "quant", "rows": 1, "cols": 30000017, "x": "f32", "out": "f32", "both": False, "stochastic": True},
        # activations of a training step, needed along both axes (forward and weight gradient)
        {"name": "mx_both_axes", "op": "quant", "rows": 8192, "cols": 5120, "x": "bf16", "out": "bf16", "both": True, "stochastic": False},
        # serving: a single token through a 4-bit layer
        {"name": "mx_linear_one_token", "op": "linear", "M": 1, "K": 4096, "N": 12288, "train": False},
        # serving: a prompt
        {"name": "mx_linear_prompt", "op": "linear", "M": 4096, "K": 8192, "N": 8192, "train": False},
        # training: ragged number of tokens, odd widths; output and both gradients
        {"name": "mx_linear_train_ragged", "op": "linear", "M": 3001, "K": 2050, "N": 5003, "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adamw", "adamw", "quant", "linear"])
    if kind == "adamw":
        bits, g = rng.choice([32, 8]), rng.choice(["f32", "bf16", "mx"])
        p = rng.choice(["f32", "f32", "bf16"])
        sizes = rng.choice(["ragged:%d:%d" % (_log(rng, 1, 600), _log(rng, 20, 40000)), "block:%d:%d:%d" % (_log(rng, 33, 1600), _log(rng, 65, 4400), rng.randint(1, 2))])
        return {"op": "adamw", "bits": bits, "p": p, "g": g, "K": rng.choice([1, 1, 2, 3, 5, 8]), "sizes": sizes,
                "shadow": p == "f32" and rng.random() < 0.5, "pad": bits == 8 or g == "mx" or rng.random() < 0.5}
    if kind == "quant":
        rows = rng.choice([1, _log(rng, 2, 9000)])
        x = rng.choice(["f32", "bf16"])
        return {"op": "quant", "rows": rows, "cols": _log(rng, 1, 20000000 if rows == 1 else 4500), "x": x, "out": x, "both": rows > 1 and rng.random() < 0.5,
                "stochastic": rng.random() < 0.5}
    return {"op": "linear", "M": _log(rng, 1, 3000), "K": _log(rng, 32, 5000), "N": _log(rng, 16, 5000), "train": rng.random() < 0.5}


def _sizes(case):
    """Lengths of the tensors of an AdamW case."""
    s = case["sizes"]
    if s.startswith("ragged:"):
        n, top = (int(v) for v in s.split(":")[1:])
        return [1 + (i * 7919 + 13 * i * i) % top for i in range(n)]
    if s.startswith("block:"):
        d, f, n = (int(v) for v in s.split(":")[1:])
        return [d * d, d * d, d * d, d * d, d * f, d * f, f * d, d, d] * n
    return [int(v) for v in s.split(",")]


def _offsets(case):
    sizes, at, out = _sizes(case), 0, []
    for n in sizes:
        out.append(at)
        at += (n + 31) // 32 * 32 if case["pad"] else n
    return sizes, out, at


# ---- random numbers of stochastic rounding (inputs of both forms) -----------------------------------------------------
def _philox(key, c0, c1, c2, c3):
    """Philox4x32-10 on int64 tensors that hold 32-bit words."""
    k0, k1 = key & 0xFFFFFFFF, (key >> 32) & 0xFFFFFFFF

    def mul(a, x):
        p0, p1 = a * (x & 0xFFFF), a * (x >> 16)
        return (p1 + (p0 >> 16)) >> 16, (p0 + ((p1 & 0xFFFF) << 16)) & 0xFFFFFFFF

    for _ in range(10):
        h0, l0 = mul(0xD2511F53, c0)
        h1, l1 = mul(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c0, c1, c2, c3


def _halves(words):
    """Four words per group -> eight 16-bit numbers per group: low half, then high half of each word."""
    w = torch.stack(words, -1)
    return torch.stack([w & 0xFFFF, w >> 16], -1).flatten(-3).to(torch.int32)


def _state_bits16(case, seed):
    """The 16-bit number of every element of the flat buffer: counter = (group of eight in its tensor, tag 2, step, tensor)."""
    sizes, offs, total = _offsets(case)
    ends = torch.tensor(offs + [total], device=DEV)
    group = torch.arange(total // 8, device=DEV)
    tensor = torch.searchsorted(ends, group * 8, right=True) - 1
    inside = group - ends[tensor] // 8
    return _halves(_philox(seed, inside & 0xFFFFFFFF, (2 << 24) | (inside >> 32), torch.full_like(group, STEP), tensor))


def _quant_bits16(rows, cols, seed, tag):
    """The same for quantisation: counter = (group of eight in its row, tag, row, row >> 32)."""
    g = torch.arange((cols + 7) // 8, device=DEV)
    r = torch.arange(rows, device=DEV)
    c0, c2 = g.expand(rows, -1).contiguous(), r[:, None].expand(-1, g.numel()).contiguous()
    u = _halves(_philox(seed, c0, torch.full_like(c0, tag << 24), c2, torch.zeros_like(c0)))
    return u.view(rows, -1)[:, :cols]


# ---- plain forms, 32 bits -----------------------------------------------------------------------------------------------
def _exponent(top, limit_bits):
    """Smallest k with top <= L * 2^k, L = 6 (limit_bits 1.5, 2) or 448 (1.75, 8); the lowest exponent where top is zero."""
    frac, emax = limit_bits
    f, e = torch.frexp(top)
    k = e - 1 - emax + (2 * f > frac).to(e.dtype)
    return torch.where(top > 0, k, torch.full_like(k, -127)).clamp(min=-127)


E2M1, E4M3 = (1.5, 2), (1.75, 8)


def _pow2(k):
    """2^k in 32 bits, -127 <= k <= 127, from its bits (2^-127 is subnormal)."""
    k = k.to(torch.int32)
    return torch.where(k > -127, (k + 127) << 23, torch.full_like(k, 1 << 22)).view(torch.float32)


def _blocks(x):
    """[rows, cols] -> [rows, blocks, 32], zeros behind the end."""
    pad = -x.shape[-1] % 32
    return torch.nn.functional.pad(x, (0, pad)).unflatten(-1, (-1, 32))


def _mx_plain(x, u=None):
    """(grid values in units of the scale, exponents): the MXFP4 form of the rows of x."""
    b = _blocks(x.float())
    k = _exponent(b.abs().amax(-1), E2M1)
    a = b.abs() * _pow2(-k)[..., None]
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.round(a / step) if u is None else torch.floor((a / step).double() + _blocks(u).double() * 2.0**-16).float()   # 64 bits: the sum may lie next to a whole number
    return torch.copysign(q * step, b), k


def _mx_value(q, k, cols):
    return (q * _pow2(k)[..., None]).flatten(-2)[..., :cols]


def _e4m3_plain(x, u, keep):
    """E4M3 values and exponents of non-empty blocks of 32 under stochastic rounding; keep: a positive value stays positive."""
    b = x.view(-1, 32)
    k = _exponent(b.abs().amax(-1), E4M3)
    a = b.abs() * _pow2(-k)[:, None]
    step = _pow2((torch.frexp(a)[1] - 1).clamp(min=-6) - 3)
    q = torch.floor(a / step + u.view(-1, 32).float() * 2.0**-16) * step
    if keep:
        q = torch.where((a > 0) & (q == 0), torch.full_like(q, 2.0**-9), q)
    return torch.copysign(q, b), k


def _swap_bytes(u):
    return ((u & 0xFF) << 8) | (u >> 8)


def _codes_e4m3(q, k):
    return q.to(torch.float8_e4m3fn).view(-1), (k + 127).to(torch.uint8)


def _adamw_plain(s):
    case, c = s["case"], s["step"]
    g = s["g"][0].float() if case["g"] != "mx" else _mx_decode(s["g"][0], s["g_scale"][0])
    for more in range(1, case["K"]):
        g = g + (s["g"][more].float() if case["g"] != "mx" else _mx_decode(s["g"][more], s["g_scale"][more]))
    g = g / case["K"]
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, 32) * _pow2(s["m_scale"].int() - 127)[:, None]).view(-1)
        r = (s["v"].float().view(-1, 32) * _pow2(s["v_scale"].int() - 127)[:, None]).view(-1)
        v = r * r
    m = BETAS[0] * m + (1 - BETAS[0]) * g
    v = BETAS[1] * v + (1 - BETAS[1]) * g * g
    r = torch.sqrt(v)
    p = s["p"].float()
    p = p * (1 - LR * DECAY) - LR / (1 - BETAS[0] ** c) * m / (r / math.sqrt(1 - BETAS[1] ** c) + EPS)
    s["p"].copy_(p)
    if case["shadow"]:
        s["shadow"].copy_(p)
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        q, k = _codes_e4m3(*_e4m3_plain(m, s["u"], False))
        s["m"].copy_(q)
        s["m_scale"].copy_(k)
        q, k = _codes_e4m3(*_e4m3_plain(r, _swap_bytes(s["u"]), True))
        s["v"].copy_(q)
        s["v_scale"].copy_(k)


_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx_decode(codes, scales):
    """Flat vector of MXFP4: two codes a byte (low half first), one scale byte per 32 elements."""
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), device=codes.device)
    v = grid[torch.stack([codes & 15, codes >> 4], -1).view(-1).int()]
    return (v.view(-1, 32) * _pow2(scales.int() - 127)[:, None]).view(-1)


def _pack(q, k):
    """Codes two a byte and scale bytes of grid values q [rows, blocks, 32] and exponents k, rows padded to 128 elements."""
    code = torch.bucketize(q.abs(), torch.tensor(_GRID, device=q.device)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    code = code.flatten(-2)
    code = torch.nn.functional.pad(code, (0, -code.shape[-1] % 128))
    return code[..., 0::2] | (code[..., 1::2] << 4), (k + 127).to(torch.uint8)


def _tiles(scales):
    """Scale bytes [rows, blocks] in the order the products read them: tiles of 128 rows x 4 blocks, 512 bytes each, row r of
    a tile at byte 16 (r % 32) + 4 (r / 32)."""
    r, b = scales.shape
    s = torch.nn.functional.pad(scales, (0, -b % 4, 0, -r % 128))
    s = s.view(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4)
    return s.contiguous().view(-1)


# ---- inputs -------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)

    s = {"case": case, "seed": seed * 2654435761 % (1 << 48) + 7, "step": STEP}
    if case["op"] == "quant":
        x = normal(case["rows"], case["cols"])
        s["x"] = (x * torch.exp(0.7 * normal(case["rows"], 1)) * (1e-3 if case["stochastic"] else 1.0)).to(DTYPES[case["x"]])
        if not own and case["stochastic"]:
            s["u"] = _quant_bits16(case["rows"], case["cols"], s["seed"], 3)
            s["ut"] = _quant_bits16(case["cols"], case["rows"], s["seed"], 4) if case["both"] else None
        return s
    if case["op"] == "linear":
        s["x"] = normal(case["M"], case["K"]).to(torch.bfloat16)
        w = (normal(case["N"], case["K"]) / math.sqrt(case["K"])).to(torch.bfloat16)
        if case["train"]:
            s["w"], s["dy"] = w, (normal(case["M"], case["N"]) * 1e-2).to(torch.bfloat16)
            if not own:
                s["u"] = _quant_bits16(case["M"], case["N"], s["seed"], 3)
                s["ut"] = _quant_bits16(case["N"], case["M"], s["seed"], 4)
        else:   # a served layer keeps its weights in 4 bits
            q, k = _mx_plain(w)
            s["w_codes"], lin = _pack(q, k)
            s["w_linear"], s["w_scales"] = lin, _tiles(lin)
        return s
    sizes, offs, n = _offsets(case)
    live = torch.zeros(n, dtype=torch.bool, device=DEV)
    ends = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    ends.index_add_(0, torch.tensor(offs, device=DEV), torch.ones(len(offs), dtype=torch.int32, device=DEV))
    ends.index_add_(0, torch.tensor([o + c for o, c in zip(offs, sizes)], device=DEV), -torch.ones(len(offs), dtype=torch.int32, device=DEV))
    live = torch.cumsum(ends, 0)[:n] > 0
    del ends
    spread = torch.exp(0.5 * normal(n // 32 + 1)).repeat_interleave(32)[:n] * 1e-3 * live
    s["p"] = (0.02 * normal(n) * live).to(DTYPES[case["p"]])
    s["g"], s["g_scale"] = [], []
    for _ in range(case["K"]):
        g = normal(n) * spread
        if case["g"] == "mx":
            codes, scales = _pack(*_mx_plain(g.view(1, -1)))
            s["g"].append(codes.view(-1)[: n // 2])
            s["g_scale"].append(scales.view(-1))
        else:
            s["g"].append(g.to(DTYPES[case["g"]]))
    m, r = 0.3 * normal(n) * spread, spread * (0.7 + 0.1 * normal(n).abs())
    if case["bits"] == 32:
        s["m"], s["v"] = m, r * r
    else:
        half = torch.full((n,), 1 << 15, dtype=torch.int32, device=DEV)
        s["m"], s["m_scale"] = _codes_e4m3(*_e4m3_plain(m, half, False))
        s["v"], s["v_scale"] = _codes_e4m3(*_e4m3_plain(r, half, True))
    if case["shadow"]:
        s["shadow"] = s["p"].to(torch.bfloat16)
    if own:
        from paper_2003_10579_b200 import binding as B

        def views(t, per=1):
            return [t[o // per: o // per + -(-c // per)] for o, c in zip(offs, sizes)]

        if case["g"] == "mx":
            grads = [[B.MxTensor(a, b, 1, c, "linear") for a, b, c in zip(views(g, 2), views(k, 32), sizes)] for g, k in zip(s["g"], s["g_scale"])]
        else:
            grads = [views(g) for g in s["g"]]
        state = {"m": views(s["m"]), "v": views(s["v"])}
        if case["bits"] == 8:
            state = {"m": views(s["m"].view(torch.uint8)), "v": views(s["v"].view(torch.uint8)), "m_scale": views(s["m_scale"], 32), "v_scale": views(s["v_scale"], 32)}
        s["opt"] = B.AdamW(views(s["p"]), grads, betas=BETAS, eps=EPS, weight_decay=DECAY, state_bits=case["bits"], state=state,
                           shadow=views(s["shadow"]) if case["shadow"] else None, seed=s["seed"])
    elif case["bits"] == 8:
        s["u"] = _state_bits16(case, s["seed"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        from paper_2003_10579_b200 import binding as B
    if case["op"] == "adamw":
        if own:
            s["opt"].step(s["step"], LR)
        else:
            _adamw_plain(s)
        out = {k: s[k] for k in ("p", "shadow", "m", "v") if k in s}
        if case["bits"] == 8:
            out["m_scale"], out["v_scale"] = s["m_scale"].view(torch.float8_e8m0fnu), s["v_scale"].view(torch.float8_e8m0fnu)
        return out
    if case["op"] == "quant":
        dt, sr = DTYPES[case["out"]], case["stochastic"]
        if own:
            q = B.mx_quantize(s["x"], along="both" if case["both"] else "rows", rounding="stochastic" if sr else "nearest", seed=s["seed"],
                              layout="tiles" if case["both"] else "linear")
            return [B.mx_dequantize(t, dt) for t in (q if case["both"] else (q,))]
        rows, cols = case["rows"], case["cols"]
        out = [_mx_value(*_mx_plain(s["x"], s["u"] if sr else None), cols).to(dt)]
        if case["both"]:
            out.append(_mx_value(*_mx_plain(s["x"].t(), s["ut"] if sr else None), rows).to(dt))
        return out
    M, N, K = case["M"], case["N"], case["K"]
    if not case["train"]:
        if own:
            w = B.MxTensor(s["w_codes"], s["w_scales"], N, K, "tiles")
            return B.mx_matmul(B.mx_quantize(s["x"]), w, torch.bfloat16)
        w = _mx_decode_rows(s["w_codes"], s["w_linear"], K)
        return (_mx_value(*_mx_plain(s["x"]), K) @ w.t()).to(torch.bfloat16)
    # training: y = x w^T, dx = dy w, dw = dy^T x; gradients rounded stochastically, the rest to nearest
    if own:
        x, xt = B.mx_quantize(s["x"], along="both")
        w, wt = B.mx_quantize(s["w"], along="both")
        dy, dyt = B.mx_quantize(s["dy"], along="both", rounding="stochastic", seed=s["seed"])
        return {"y": B.mx_matmul(x, w, torch.bfloat16), "dx": B.mx_matmul(dy, wt, torch.bfloat16), "dw": B.mx_matmul(dyt, xt, torch.float32)}
    x, xt = _mx_value(*_mx_plain(s["x"]), K), _mx_value(*_mx_plain(s["x"].t()), M)
    w, wt = _mx_value(*_mx_plain(s["w"]), K), _mx_value(*_mx_plain(s["w"].t()), N)
    dy, dyt = _mx_value(*_mx_plain(s["dy"], s["u"]), N), _mx_value(*_mx_plain(s["dy"].t(), s["ut"]), M)
    return {"y": (x @ w.t()).to(torch.bfloat16), "dx": (dy @ wt.t()).to(torch.bfloat16), "dw": dyt @ xt.t()}


def _mx_decode_rows(codes, scales, cols):
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), device=codes.device)
    v = grid[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    b = scales.shape[1]
    return (v[:, : 32 * b].unflatten(1, (b, 32)) * _pow2(scales.int() - 127)[..., None]).flatten(1)[:, :cols]


# ---- work and exact values ----------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        state = 16.0 if case["bits"] == 32 else 4.0 + 4.0 / 32
        return {"bytes": n * (2 * BYTES[case["p"]] + case["K"] * BYTES[case["g"]] + state + (2 if case["shadow"] else 0)), "flops": n * (14.0 + case["K"])}
    if case["op"] == "quant":
        n, ways = case["rows"] * case["cols"], 2 if case["both"] else 1
        return {"bytes": n * (BYTES[case["x"]] + ways * BYTES[case["out"]]), "flops": 4.0 * n * ways}
    M, N, K = case["M"], case["N"], case["K"]
    if case["train"]:
        return {"bytes": 2.0 * (M * K + N * K + 2 * M * N + M * K) + 4.0 * N * K, "flops": 6.0 * M * N * K}
    return {"bytes": 2.0 * M * K + N * K * BYTES["mx"] + 2.0 * M * N, "flops": 2.0 * M * N * K}


def _round64(x, grid, emax_limit, u=None, keep=False):
    """Rows of blocks of 32 in 64 bits against the list of a format's non-negative values: nearest (ties to the even place in
    the list) or stochastic (from the two neighbours).  Returns values in units of the scale, and the scale."""
    grid = torch.tensor(grid, dtype=torch.float64, device=x.device)
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, torch.ones_like(top)) / emax_limit)).clamp(min=-127))
    scale = torch.where(scale * emax_limit < top, scale * 2, scale)
    scale = torch.where(scale * emax_limit / 2 >= top, scale / 2, scale)
    scale = torch.where(top > 0, scale.clamp(min=2.0**-127), torch.full_like(scale, 2.0**-127))
    a = x.abs() / scale
    lo = (torch.searchsorted(grid, a, right=True) - 1).clamp(max=len(grid) - 1)
    hi = (lo + 1).clamp(max=len(grid) - 1)
    gap = torch.where(hi > lo, grid[hi] - grid[lo], torch.ones_like(a))
    part = (a - grid[lo]) / gap
    if u is None:
        up = (part > 0.5) | ((part == 0.5) & (lo % 2 == 1))
    else:
        up = part + u.double() / 65536 >= 1
    q = torch.where(up, grid[hi], grid[lo])
    if keep:
        q = torch.where((q == 0) & (a > 0), grid[1], q)
    return torch.where(x < 0, -q, q), scale


def _mx64(x, u=None):
    cols = x.shape[1]
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for at in range(0, x.shape[0], max(1, 40000000 // cols)):   # a slab of rows at a time: 64-bit copies are large
        rows = slice(at, at + max(1, 40000000 // cols))
        b = torch.nn.functional.pad(x[rows].double(), (0, -cols % 32)).unflatten(1, (-1, 32))
        uu = None if u is None else torch.nn.functional.pad(u[rows], (0, -cols % 32)).unflatten(1, (-1, 32))
        q, scale = _round64(b, _GRID, 6.0, uu)
        out[rows] = (q * scale).flatten(1)[:, :cols]
    return out


_E4M3_GRID = [i * 2.0**-9 for i in range(8)] + [(8 + i) * 2.0**(e - 10) for e in range(1, 16) for i in range(8)][:-1]
assert _E4M3_GRID[-1] == 448.0


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        n = s["p"].numel()
        out = {"p": torch.empty(n, dtype=torch.float64, device=DEV), "m": torch.empty(n, dtype=torch.float64, device=DEV), "v": torch.empty(n, dtype=torch.float64, device=DEV)}
        scales = {"m_scale": torch.empty(-(-n // 32), dtype=torch.float64, device=DEV), "v_scale": torch.empty(-(-n // 32), dtype=torch.float64, device=DEV)}
        for at in range(0, n, 1 << 25):
            here, blocks = slice(at, min(n, at + (1 << 25))), slice(at // 32, -(-min(n, at + (1 << 25)) // 32))
            g = 0.0
            for l in range(case["K"]):
                if case["g"] == "mx":
                    c = s["g"][l][here.start // 2: here.stop // 2].long()
                    c = torch.stack([c % 16, c // 16], 1).view(-1)
                    mag = torch.tensor(_GRID, dtype=torch.float64, device=DEV)[c % 8] * (1 - 2 * (c // 8))
                    g = g + mag * torch.exp2(s["g_scale"][l][blocks].double() - 127).repeat_interleave(32)
                else:
                    g = g + s["g"][l][here].double()
            g = g / case["K"]
            m, v = s["m"][here].double(), s["v"][here].double()
            if case["bits"] == 8:
                m = m * torch.exp2(s["m_scale"][blocks].double() - 127).repeat_interleave(32)
                v = (v * torch.exp2(s["v_scale"][blocks].double() - 127).repeat_interleave(32)) ** 2
            m, v = m + (1 - BETAS[0]) * (g - m), v + (1 - BETAS[1]) * (g * g - v)
            mh, vh = m / (1 - BETAS[0] ** STEP), v / (1 - BETAS[1] ** STEP)
            p = s["p"][here].double()
            out["p"][here] = p - LR * (mh / (vh.sqrt() + EPS) + DECAY * p)
            if case["bits"] == 8:
                u = s["u"][here].view(-1, 32)
                q, k = _round64(m.view(-1, 32), _E4M3_GRID, 448.0, u)
                out["m"][here], scales["m_scale"][blocks] = q.view(-1), k.view(-1)
                q, k = _round64(v.sqrt().view(-1, 32), _E4M3_GRID, 448.0, u % 256 * 256 + u // 256, True)
                out["v"][here], scales["v_scale"][blocks] = q.view(-1), k.view(-1)
            else:
                out["m"][here], out["v"][here] = m, v
        if case["shadow"]:
            out["shadow"] = out["p"]
        return {**out, **scales} if case["bits"] == 8 else out
    if case["op"] == "quant":
        out = [_mx64(s["x"], s.get("u"))]
        return out + [_mx64(s["x"].t(), s.get("ut"))] if case["both"] else out
    if not case["train"]:
        c = s["w_codes"].long()
        c = torch.stack([c % 16, c // 16], -1).flatten(1)
        mag = torch.tensor(_GRID, dtype=torch.float64, device=DEV)[c % 8] * (1 - 2 * (c // 8))
        scale = torch.exp2(s["w_linear"].double() - 127).repeat_interleave(32, 1)
        w = (mag[:, : scale.shape[1]] * scale)[:, : case["K"]]
        return _mx64(s["x"]) @ w.t()
    x, xt, w, wt = _mx64(s["x"]), _mx64(s["x"].t()), _mx64(s["w"]), _mx64(s["w"].t())
    dy, dyt = _mx64(s["dy"], s["u"]), _mx64(s["dy"].t(), s["ut"])
    return {"y": x @ w.t(), "dx": dy @ wt.t(), "dw": dyt @ xt.t()}
