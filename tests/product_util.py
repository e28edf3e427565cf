"""64-bit plain forms of the operators that multiply by stored codes, and bounds of their errors.

Bounds.  A matrix step adds at most 17 numbers (16 exact products, or 32 in 8 bits, and the sum so far); each addend loses
less than 2^-24 of the largest when they are aligned, the sum is cut once, so a step is off by less than 2^-19 of the sum
S of the products' magnitudes (33 addends of 2^-24).  Steps: k / 16; a few more additions join the warps and blocks.  A result is
then rounded by at most half a step of its type, torch.finfo(dtype).eps / 2 of it."""
import numpy as np
import torch

from oracle import mxq_oracle as orc


def sum_bound(k: int, magnitudes):
    return (k / 16 + 16) * 2.0 ** -19 * magnitudes


def value_table(fmt: str) -> np.ndarray:
    """Element value of each code of a format, from the definition: sign, exponent and mantissa fields, or two's complement."""
    bits = orc.bits(fmt)
    if fmt.startswith("int"):
        c = np.arange(1 << bits)
        return np.where(c >= 1 << (bits - 1), c - (1 << bits), c).astype(np.float64)
    eta, mu = int(fmt[1]), int(fmt[3])
    out = []
    for c in range(1 << bits):
        e, f = (c >> mu) & ((1 << eta) - 1), c & ((1 << mu) - 1)
        bias = (1 << (eta - 1)) - 1
        v = f * 2.0 ** (1 - bias - mu) if e == 0 else (1 + f / (1 << mu)) * 2.0 ** (e - bias)
        out.append(-v if c >> (bits - 1) else v)
    return np.array(out)


def scale64(b) -> np.ndarray:
    b = np.asarray(b).astype(np.int64)
    return np.where(b == 255, np.nan, np.ldexp(1.0, b - 127))


def values64(codes: np.ndarray, scales: np.ndarray, fmt: str, block: int) -> np.ndarray:
    """Unpacked codes [..., k] and scale bytes [..., k / block] -> their values."""
    with np.errstate(invalid="ignore"):
        return value_table(fmt)[codes] * np.repeat(scale64(scales), block, axis=-1)


def quantized(rng, rows: int, k: int, fmt: str, block: int, std: float = 1.0):
    """A random operand through the oracle: (packed codes, scales [rows, k / block], values in 64 bits)."""
    x = (rng.standard_normal((rows, k)) * std * np.exp2(rng.integers(-4, 5, (rows, 1)))).astype(np.float32)
    codes, scales = orc.quantize(x.reshape(-1), fmt, block)
    packed = orc.pack(codes, orc.bits(fmt))
    mask = (1 << orc.bits(fmt)) - 1
    codes = (np.asarray(codes).astype(np.int64) & mask).reshape(rows, k)
    scales = np.asarray(scales).reshape(rows, k // block)
    return np.asarray(packed), scales, values64(codes, scales, fmt, block)


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def to64(t: torch.Tensor) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def check(got: torch.Tensor, want: np.ndarray, bound: np.ndarray):
    """got is within `bound` plus its type's rounding of `want`; NaN exactly where want is."""
    g = to64(got)
    assert g.shape == want.shape
    assert np.array_equal(np.isnan(g), np.isnan(want))
    fine = np.isfinite(want)
    lim = bound[fine] + (half_step(got.dtype) * (np.abs(want[fine]) + bound[fine])) + np.finfo(np.float32).tiny
    err = np.abs(g[fine] - want[fine])
    worst = float((err / lim).max()) if err.size else 0.0
    assert worst <= 1.0, "off by %.3g of the bound" % worst


def padded64(v: np.ndarray, block: int) -> np.ndarray:
    return np.pad(v, ((0, 0), (0, -v.shape[1] % block)))


def e4m3_64(v: np.ndarray, block: int) -> np.ndarray:
    """Values of FP32-representable v after MXFP8 E4M3 along the rows (padded), through the oracle."""
    p = padded64(v, block).astype(np.float32)
    codes, scales = orc.quantize(np.ascontiguousarray(p).reshape(-1), "e4m3", block)
    return values64(np.asarray(codes).astype(np.int64).reshape(p.shape), np.asarray(scales).reshape(p.shape[0], -1), "e4m3", block)


def choice64(logits: np.ndarray, top_k: int, renormalize: bool):
    """Per token [(expert, weight)]: the largest logits, ties to the lowest index, -inf never."""
    out = []
    for row in logits.astype(np.float64):
        if np.isnan(row).any():
            out.append(None)
            continue
        order = [e for e in sorted(range(row.size), key=lambda e: (-row[e], e)) if row[e] > -np.inf][:top_k]
        if not order:
            out.append([])
            continue
        p = np.exp(row - row[order[0]])
        total = p[order].sum() if renormalize else p.sum()
        out.append([(e, p[e] / total) for e in order])
    return out


def moe64(x, logits, up, down, inner, top_k, renormalize, dtype):
    """The layer in 64 bits and the bound of a kernel's error (see the module's note): h from sums of `hidden` products, kept
    to 16 bits (24 for FP32), then sums of `inner` products; silu's slope is below 1.1, exp and the division are good to 2^-20."""
    t, hidden = x.shape
    out, bound = np.zeros((t, hidden)), np.zeros((t, hidden))
    kept = 2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -23
    for i, chosen in enumerate(choice64(logits, top_k, renormalize)):
        if chosen is None:
            out[i] = np.nan
            continue
        for e, w in chosen:
            gu, mag = up[e] @ x[i], np.abs(up[e]) @ np.abs(x[i])
            off = sum_bound(hidden, mag)
            g, u = gu[:inner], gu[inner:]
            with np.errstate(over="ignore"):
                s = g / (1 + np.exp(-g))
            h = s * u
            dh = 1.1 * off[:inner] * (np.abs(u) + off[inner:]) + np.abs(s) * off[inner:] + (kept + 2.0 ** -20) * np.abs(h)
            out[i] += w * (down[e] @ h)
            a = np.abs(down[e])
            bound[i] += w * (a @ dh + sum_bound(inner, a @ (np.abs(h) + dh)) + 2.0 ** -20 * (a @ np.abs(h)))
    return out, bound
