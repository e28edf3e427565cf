"""How exact FP32 results of the products are, next to what their sums in 32 bits allow; and inputs for which that shows.

norm_limit: a product over k is summed in k / 32 steps (or in fewer, parts of them side by side).  The matrix instruction cuts the sum of each
step to FP32, toward zero: it loses less than 2^-23 of the sum so far.  Cuts of one sum do not cancel, they add up; and for terms
of random sign the sum so far after i of N steps is sqrt(i / N) of the result in size, so that the losses come to less than
2^-23 sum_i sqrt(i / N) = 2/3 N 2^-23 of the result in norm, to half of that on average.  (Steps that rounded to nearest would come to
2^-24 sqrt(N / 2), 9e-7 for k = 14336, and the instruction does not: 8.4e-6 there, a quarter of it where k is summed in four
parts.  Where a step's sum has no bits to cut, as with blocks of one scale, nothing is lost.)  A result rounded to BF16 once is off by
about 2^-9.3 in norm, partial sums rounded to FP16 by 2^-12.

one_product: tokens with one element that is not zero, down matrices with one such element per row: every sum of the layer
is one product, whatever the order, and its error can be counted.  In units of 2^-22 of the value: a product of an FP32 number
in three parts with a weight, summed in three steps, the first exact, the others cut: 1 for the gate, 1 for the up half, 1 for
the down matrix.  silu(g) = g / (1 + exp(-g)): the gate's error times 1 + |g| instead of 1, exp 1 (two units in the last place), its sum
with 1 and the division 1/2.  The product with the up half 1/4; three parts hold all 24 bits of it.  Together |g| + 4.75; the bound is |g| + 6.
Two parts instead of three leave 2^-16 of a token or of an inner activation out: 64 units."""
import numpy as np
import torch

from oracle import mxq_oracle as orc

import product_util as pu

FORMATS = ("e4m3", "e2m1", "int8", "int4")


def norm_limit(k: int) -> float:
    return 2 / 3 * (k / 32) * 2.0 ** -23


def norm_error(got, want) -> float:
    """||got - want|| / ||want||, of tensors."""
    return float((got.double() - want).norm() / want.norm())


def one_product(rng, fmt, tokens=32, experts=3, hidden=128, inner=64, block=32):
    """(x, logits, up codes, up scales, down codes, down scales, unpacked up and down values [e, rows, k])."""
    bits, table = orc.bits(fmt), pu.value_table(fmt)
    usable = np.flatnonzero(np.abs(table) < 450)            # (E4M3's NaN codes stand at 480 in the table)
    scale = 127 + int(np.floor(np.log2(2.0 / np.abs(table[usable]).max())))
    x = np.zeros((tokens, hidden), np.float32)
    at = rng.integers(0, hidden, tokens)
    x[np.arange(tokens), at] = rng.uniform(0.5, 1.0, tokens).astype(np.float32) * rng.choice([-1.0, 1.0], tokens).astype(np.float32)
    up = rng.choice(usable, (experts, 2 * inner, hidden))
    down = np.zeros((experts, hidden, inner), np.int64)
    rows = np.arange(hidden)
    down[:, rows, rows % inner] = rng.choice(usable[np.abs(table[usable]) >= 1], (experts, hidden))
    logits = np.full((tokens, experts), -np.inf, np.float32)
    logits[np.arange(tokens), np.arange(tokens) % experts] = 1.0
    packed = [orc.pack(c.reshape(-1).astype(np.uint8), bits) for c in (up, down)]
    scales = [np.full(c.size // block, scale, np.uint8) for c in (up, down)]
    values = [table[c] * 2.0 ** (scale - 127) for c in (up, down)]
    return x, logits, packed[0], scales[0], packed[1], scales[1], values[0], values[1]


def one_product64(x, logits, up, down, keep_x=lambda v: v, keep_h=lambda v: v):
    """The layer in 64 bits and its bound; keep_x, keep_h: what is left of a token and of an inner activation."""
    inner = down.shape[2]
    out, bound = np.zeros(x.shape), np.zeros(x.shape)
    for t, e in enumerate(np.argmax(logits, 1)):
        gu = up[e] @ keep_x(x[t].astype(np.float64))
        g, h = gu[:inner], keep_h(gu[:inner] / (1 + np.exp(-gu[:inner])) * gu[inner:])
        out[t] = down[e] @ h
        which = np.arange(out.shape[1]) % inner
        bound[t] = (np.abs(g[which]) + 6) * 2.0 ** -22 * np.abs(out[t]) + np.finfo(np.float32).tiny
    return out, bound


def bf16_parts(v, parts: int):
    """v as the sum of `parts` BF16 numbers, each but the last cut, the last rounded to nearest, as 64-bit values."""
    left, total = np.asarray(v, np.float64).astype(np.float32), 0.0
    for i in range(parts):
        if i + 1 < parts:
            part = (left.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
        else:
            part = torch.from_numpy(left.copy()).bfloat16().float().numpy()
        total, left = total + part.astype(np.float64), left - part
    return total
