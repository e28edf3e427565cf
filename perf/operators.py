"""The products of a network whose weights are held in microscaling formats, as cases that can be timed.

Four operators that read or write the library's codes and scales:

  matmul            D = A^ B^T of two MXFP8 E4M3 operands [m, k] and [n, k], one scale per block along k
  quantize_matrix   MXFP8 E4M3 codes of a matrix along its rows and of its transpose from one read: what the three
                    products of a training step take
  linear_ste        y = Q(x) Q(w)^T inside autograd, with dx = Q(dy) Q(w^T)^T and dw = Q(dy^T) Q(x^T)^T
  moe               a mixture-of-experts layer for a few tokens over experts held as codes: routing from the
                    router's logits, gated products, weighted sum

The plain forms below are written from these formulas in elementary torch operations, in 32 bits, and rounded once
to the output's type.  Widths are those of the 8B Llama-shaped weight set (4096, 14336, 1024) or generic ones.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
#: format -> (bits, exponent bits, mantissa bits); exponent bits 0: two's complement integers
FMT = {"e4m3": (8, 4, 3), "e2m1": (4, 2, 1), "int8": (8, 0, 0), "int4": (4, 0, 0)}


def listed():
    return [
        # one decoded token through a square projection: the smallest product there is, latency counts
        {"name": "matmul_token", "op": "matmul", "m": 1, "n": 4096, "k": 4096, "block": 128, "dtype": "bf16"},
        # a ragged batch of decoded tokens through an MLP's up projection: bound by reading the weights
        {"name": "matmul_decode_batch", "op": "matmul", "m": 13, "n": 14336, "k": 4096, "block": 128, "dtype": "bf16"},
        # a serving step of 200 sequences through the down projection: few output tiles, a long k
        {"name": "matmul_serving_step", "op": "matmul", "m": 200, "n": 4096, "k": 14336, "block": 128, "dtype": "bf16"},
        # an odd-sized prefill with the library's default block, k not a multiple of 128, accumulated in FP32
        {"name": "matmul_odd_f32", "op": "matmul", "m": 1000, "n": 1111, "k": 1120, "block": 32, "dtype": "f32"},
        # the prefill of a long prompt through the up projection: bound by the tensor cores
        {"name": "matmul_prefill", "op": "matmul", "m": 8192, "n": 14336, "k": 4096, "block": 128, "dtype": "bf16"},
        # the operands that an MLP weight's three products take, from one read of the BF16 weight
        {"name": "matrix_mlp_weight", "op": "matrix", "rows": 14336, "cols": 4096, "block": 128, "dtype": "bf16"},
        # FP32 gradients of an odd shape: both directions end inside a block
        {"name": "matrix_odd_f32", "op": "matrix", "rows": 1000, "cols": 1111, "block": 32, "dtype": "f32"},
        # forward and backward of one square projection over a batch of 4096 tokens
        {"name": "linear_step", "op": "linear", "m": 4096, "n": 4096, "k": 4096, "block": 128, "dtype": "bf16"},
        # the same for a short FP32 sequence and a head of odd width
        {"name": "linear_odd_f32", "op": "linear", "m": 333, "n": 1000, "k": 1024, "block": 32, "dtype": "f32"},
        # one decoded token, many small experts in 4 bits: latency counts
        {"name": "moe_token_small_experts", "op": "moe", "t": 1, "experts": 64, "top_k": 8, "hidden": 2048,
         "inner": 1024, "fmt": "e2m1", "block": 32, "dtype": "bf16"},
        # one decoded token, two of eight large experts in the 8-bit anchor
        {"name": "moe_token_large_experts", "op": "moe", "t": 1, "experts": 8, "top_k": 2, "hidden": 4096,
         "inner": 14336, "fmt": "e4m3", "block": 128, "dtype": "bf16"},
        # a batch of 32 decoded tokens: nearly every expert is read, each by a few tokens
        {"name": "moe_batch_int8", "op": "moe", "t": 32, "experts": 64, "top_k": 8, "hidden": 2048, "inner": 1024,
         "fmt": "int8", "block": 32, "dtype": "bf16"},
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    def log_step(lo, hi, step):
        return step * log_int(max(1, lo // step), hi // step)

    op = rng.choice(["matmul", "matmul", "matmul", "matrix", "linear", "moe", "moe"])
    block = rng.choice([32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "matmul":
        return {"op": op, "m": log_int(1, 8192), "n": log_int(64, 14336), "k": log_step(512, 4096, block), "block": block,
                "dtype": dtype}
    if op == "matrix":
        return {"op": op, "rows": log_int(1, 14336), "cols": log_int(64, 4096), "block": block, "dtype": dtype}
    if op == "linear":
        return {"op": op, "m": log_int(1, 4096), "n": log_int(64, 4096), "k": log_int(64, 4096), "block": block,
                "dtype": dtype}
    experts = log_int(2, 64)
    return {"op": op, "t": log_int(1, 32), "experts": experts, "top_k": min(experts, rng.randint(1, 8)),
            "hidden": log_step(512, 2048, block), "inner": log_step(256, 1024, block), "fmt": rng.choice(sorted(FMT)),
            "block": block, "dtype": dtype}


# ---- inputs ---------------------------------------------------------------------------------------------------


def _activations(g, rows, cols, dtype):
    """N(0, 1) with 1 % of the channels 20 times as large, as a decoder's activations have them."""
    loud = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    return (torch.randn(rows, cols, generator=g, device="cuda") * loud).to(dtype)


def _weights(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda") * 0.02


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    op, block = case["op"], case["block"]
    if op == "matmul":
        a = _quantize(_activations(g, case["m"], case["k"], torch.bfloat16).float(), "e4m3", block)
        b = _quantize(_weights(g, case["n"], case["k"]), "e4m3", block)
        return {**case, "dtype": dtype, "a": a, "b": b}
    if op == "matrix":
        return {**case, "dtype": dtype, "x": _weights(g, case["rows"], case["cols"]).to(dtype)}
    if op == "linear":
        x = _activations(g, case["m"], case["k"], dtype).requires_grad_()
        w = _weights(g, case["n"], case["k"]).to(dtype).requires_grad_()
        dy = (torch.randn(case["m"], case["n"], generator=g, device="cuda") * 1e-3).to(dtype)
        return {**case, "dtype": dtype, "x": x, "w": w, "dy": dy}
    e, h, i = case["experts"], case["hidden"], case["inner"]
    return {**case, "dtype": dtype, "x": _activations(g, case["t"], h, dtype),
            "logits": torch.randn(case["t"], e, generator=g, device="cuda") * 2,
            "up": _pack(*_quantize(_weights(g, e, 2 * i, h), case["fmt"], block), case["fmt"]),
            "down": _pack(*_quantize(_weights(g, e, h, i), case["fmt"], block), case["fmt"])}


# ---- the plain forms ------------------------------------------------------------------------------------------


def _magnitudes(fmt):
    """The non-negative values of an MXFP element format in the order of their codes."""
    bits, eta, mu = FMT[fmt]
    bias, got = 2 ** (eta - 1) - 1, []
    for c in range(2 ** (bits - 1)):
        e, m = c >> mu, c & (2 ** mu - 1)
        got.append(m * 2.0 ** (1 - bias - mu) if e == 0 else (1 + m / 2 ** mu) * 2.0 ** (e - bias))
    return got[:-1] if fmt == "e4m3" else got         # S.1111.111 is NaN in E4M3


def _power(e):
    """2^e as FP32 for whole e in [-127, 127], put together from its bits."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _quantize(v, fmt, block):
    """Codes (one byte each, in v's shape) and E8M0 bytes of FP32 values, blocks along the last dimension."""
    bits, eta, mu = FMT[fmt]
    e_max = 2 ** (eta - 1) if eta else bits - 2
    parts = v.unflatten(-1, (-1, block))
    amax = parts.abs().amax(-1, keepdim=True)
    shared = (torch.frexp(amax).exponent - 1 - e_max).clamp(-127, 127)
    shared = torch.where(amax == 0, -127, shared)
    p = parts * _power(-shared)
    if eta:
        top = _magnitudes(fmt)[-1]
        low = 2 - 2 ** (eta - 1)                       # the exponent of the smallest normal value
        step = _power((torch.frexp(p).exponent - 1).clamp(min=low) - mu)
        mag = ((p / step).round() * step).abs().clamp(max=top)
        code = torch.searchsorted(torch.tensor(_magnitudes(fmt), device=v.device), mag.contiguous())
        code = code.to(torch.uint8) | (torch.signbit(p).to(torch.uint8) << (bits - 1))
    else:
        most = 2 ** (bits - 1) - 1
        whole = (torch.floor(p.abs() + 0.5) * torch.sign(p)).clamp(-most, most)
        code = (whole.to(torch.int32) & (2 ** bits - 1)).to(torch.uint8)
    return code.flatten(-2), (shared.squeeze(-1) + 127).to(torch.uint8)


def _pack(codes, scales, fmt):
    if FMT[fmt][0] == 4:
        codes = codes[..., 0::2] | (codes[..., 1::2] << 4)
    return codes.contiguous(), scales.contiguous()


def _values(codes, fmt):
    """The values that packed codes stand for, FP32."""
    bits, eta, _ = FMT[fmt]
    if bits == 4:
        codes = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    if not eta:
        c = codes.to(torch.int8) if bits == 8 else (codes << 4).to(torch.int8) >> 4
        return c.float()
    mags = _magnitudes(fmt)
    table = mags + [math.nan] * (2 ** (bits - 1) - len(mags))
    return torch.tensor(table + [-x for x in table], device=codes.device)[codes.int()]


def _dequantize(pair, fmt, block):
    codes, scales = pair
    v = _values(codes, fmt)
    return (v.unflatten(-1, (-1, block)) * _power(scales.int() - 127).unsqueeze(-1)).flatten(-2)


def _padded(v, block):
    return torch.nn.functional.pad(v, (0, -v.shape[-1] % block))


def _rounded(v, block):
    """v's values after MXFP8 E4M3 along the last dimension, padded with zeros to whole blocks."""
    return _dequantize(_quantize(_padded(v, block), "e4m3", block), "e4m3", block)


def _route(logits, top_k, renormalize=True):
    """Weights and experts of each token: the top_k largest logits, ties to the lowest index, over their softmax."""
    order = torch.sort(logits, dim=-1, descending=True, stable=True)
    ids = order.indices[:, :top_k]
    p = torch.exp(order.values - order.values[:, :1])
    w = p[:, :top_k] / (p[:, :top_k] if renormalize else p).sum(-1, keepdim=True)
    return w, ids


def _moe(s):
    w, ids = _route(s["logits"], s["top_k"])
    x, block, fmt = s["x"].float(), s["block"], s["fmt"]
    t, k, e, i = s["t"], s["top_k"], s["experts"], s["inner"]
    if t * k <= e:                                    # the weights of the chosen experts only
        at = ids.flatten()
        up = _dequantize((s["up"][0][at], s["up"][1][at]), fmt, block)
        down = _dequantize((s["down"][0][at], s["down"][1][at]), fmt, block)
        rows = x.repeat_interleave(k, 0).unsqueeze(-1)
        gu = torch.bmm(up, rows)
        gate, lift = gu[:, :i], gu[:, i:]
        out = torch.bmm(down, gate / (1 + torch.exp(-gate)) * lift).view(t, k, -1)
        return (out * w.unsqueeze(-1)).sum(1).to(s["dtype"])
    up, down = _dequantize(s["up"], fmt, block), _dequantize(s["down"], fmt, block)
    gu = torch.matmul(x, up.transpose(1, 2))          # every expert for every token
    gate, lift = gu[..., :i], gu[..., i:]
    out = torch.bmm(gate / (1 + torch.exp(-gate)) * lift, down.transpose(1, 2))
    share = torch.zeros(t, e, device=x.device).scatter_(1, ids, w)
    return (out * share.t().unsqueeze(-1)).sum(0).to(s["dtype"])


def _as_values(codes, rows):
    return codes.view(torch.float8_e4m3fn).view(rows, -1)


def run(s):
    op, block, dtype = s["op"], s["block"], s["dtype"]
    if own:
        import paper_2604_00529_b200 as mxq
        if op == "matmul":
            return mxq.matmul(*s["a"], *s["b"], s["m"], s["n"], s["k"], block=block, dtype=dtype)
        if op == "matrix":
            codes, scales, codes_t, scales_t = mxq.quantize_matrix(s["x"], block=block)
            return {"rows": _as_values(codes, s["rows"]), "row_scales": scales.view(s["rows"], -1),
                    "cols": _as_values(codes_t, s["cols"]), "col_scales": scales_t.view(s["cols"], -1)}
        if op == "linear":
            y = mxq.linear_ste(s["x"], s["w"], block=block)
            dx, dw = torch.autograd.grad(y, (s["x"], s["w"]), s["dy"])
            return {"y": y.detach(), "dx": dx, "dw": dw}
        return mxq.moe(s["x"], s["logits"], *s["up"], *s["down"], s["inner"], s["top_k"], s["fmt"], block=block)
    if op == "matmul":
        return torch.matmul(_dequantize(s["a"], "e4m3", block), _dequantize(s["b"], "e4m3", block).t()).to(dtype)
    if op == "matrix":
        x = s["x"].float()
        codes, scales = _quantize(_padded(x, block), "e4m3", block)
        codes_t, scales_t = _quantize(_padded(x.t(), block).contiguous(), "e4m3", block)
        return {"rows": _as_values(codes, s["rows"]), "row_scales": scales, "cols": _as_values(codes_t, s["cols"]),
                "col_scales": scales_t}
    if op == "linear":
        x, w, dy = s["x"].detach().float(), s["w"].detach().float(), s["dy"].float()
        y = torch.matmul(_rounded(x, block), _rounded(w, block).t())
        dx = torch.matmul(_rounded(dy, block), _rounded(w.t().contiguous(), block).t())
        dw = torch.matmul(_rounded(dy.t().contiguous(), block), _rounded(x.t().contiguous(), block).t())
        return {"y": y.to(dtype), "dx": dx.to(dtype), "dw": dw.to(dtype)}
    return _moe(s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------


def work(case):
    op, block = case["op"], case["block"]
    size = 2 if case["dtype"] == "bf16" else 4
    if op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * (k + k // block) + m * n * size, "flops": 2 * m * n * k}
    if op == "matrix":
        r, c = case["rows"], case["cols"]
        rp, cp = -(-r // block) * block, -(-c // block) * block
        return {"bytes": r * c * size + r * (cp + cp // block) + c * (rp + rp // block), "flops": 0}
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * (m * k + n * k + m * n) * size, "flops": 6 * m * n * k}
    t, e, k, h, i = case["t"], case["experts"], case["top_k"], case["hidden"], case["inner"]
    active = e * (1 - (1 - k / e) ** t)               # experts that some token chooses, in the mean
    weights = 3 * h * i * (FMT[case["fmt"]][0] / 8 + 1 / block)
    return {"bytes": active * weights + 2 * t * h * size + t * e * 4, "flops": 6 * t * k * h * i}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------


def _two_to(n):
    """2^n in 64 bits for whole n of a normal value's range."""
    return ((n.to(torch.int64) + 1023) * 2 ** 52).view(torch.float64)


def _binade(v):
    """floor(log2 |v|) of 64-bit values, from the exponent field."""
    return (v.contiguous().view(torch.int64) // 2 ** 52 % 2048 - 1023)


def _code_values64(codes, fmt):
    """Sign, exponent and mantissa fields of packed codes, put together in 64 bits."""
    bits, eta, mu = FMT[fmt]
    c = codes.to(torch.int64)
    if bits == 4:
        c = torch.stack((c % 16, c // 16), -1).flatten(-2)
    if not eta:
        return torch.where(c >= 2 ** (bits - 1), c - 2 ** bits, c).double()
    sign = 1 - 2 * (c // 2 ** (bits - 1))
    field = c // 2 ** mu % 2 ** eta
    mant = (c % 2 ** mu).double() / 2 ** mu + (field > 0)
    return sign * mant * _two_to(field.clamp(min=1) - (2 ** (eta - 1) - 1))


def _stored64(pair, fmt, block):
    v = _code_values64(pair[0], fmt)
    return v * _two_to(pair[1].to(torch.int64) - 127).repeat_interleave(block, -1)


def _e4m3_64(v, block):
    """Element values and shared exponents of E4M3 blocks along the last dimension of 64-bit values."""
    short = -v.shape[-1] % block
    if short:
        v = torch.cat((v, v.new_zeros(*v.shape[:-1], short)), -1)
    big = v.abs().reshape(*v.shape[:-1], -1, block).max(-1).values
    shared = torch.where(big > 0, _binade(big) - 8, -127).clamp(-127, 127)
    p = v / _two_to(shared).repeat_interleave(block, -1)
    grid = _two_to(_binade(p.abs().clamp(min=2.0 ** -6)) - 3)
    return torch.clamp(torch.round(p / grid) * grid, -448, 448), shared


def _rounded64(v, block):
    p, shared = _e4m3_64(v, block)
    return p * _two_to(shared).repeat_interleave(block, -1)


def exact(case, seed):
    s = prepare(case, seed)
    op, block = s["op"], s["block"]
    if op == "matmul":
        return _stored64(s["a"], "e4m3", block) @ _stored64(s["b"], "e4m3", block).T
    if op == "matrix":
        x = s["x"].double()
        return {"rows": _e4m3_64(x, block)[0], "row_scales": None, "cols": _e4m3_64(x.T.contiguous(), block)[0],
                "col_scales": None}
    if op == "linear":
        x, w, dy = s["x"].detach().double(), s["w"].detach().double(), s["dy"].double()
        return {"y": _rounded64(x, block) @ _rounded64(w, block).T,
                "dx": _rounded64(dy, block) @ _rounded64(w.T.contiguous(), block).T,
                "dw": _rounded64(dy.T.contiguous(), block) @ _rounded64(x.T.contiguous(), block).T}
    x, logits = s["x"].double(), s["logits"].double()
    out = torch.zeros(s["t"], s["hidden"], dtype=torch.float64, device=x.device)
    for token in range(s["t"]):
        row = logits[token].tolist()
        chosen = sorted(range(len(row)), key=lambda e: (-row[e], e))[:s["top_k"]]
        weight = [math.exp(row[e] - row[chosen[0]]) for e in chosen]
        for e, w in zip(chosen, weight):
            gu = _stored64((s["up"][0][e], s["up"][1][e]), s["fmt"], block) @ x[token]
            gate, lift = gu[:s["inner"]], gu[s["inner"]:]
            down = _stored64((s["down"][0][e], s["down"][1][e]), s["fmt"], block)
            out[token] += w / sum(weight) * (down @ (gate * torch.sigmoid(gate) * lift))
    return out
