"""64-bit plain forms of the operators over a paged cache of codes, and bounds of the attention's error.

Bounds.  A score is a sum of D exact products (FP32 queries: 22 bits, off by at most 2^-21 of each product) in D / 16 matrix
steps, scaled and added block by block: off by less than (D / 16 + 16) 2^-19 of the sum of the products' magnitudes (product_util).  A weight's
relative error is twice the largest score's error (the score's own and the sum's), 2^-20 for the exponential and the additions round
it, and the half step of what the weight is held in: 2^-11 (FP16) or 2^-21 (two FP16 parts).  Weights that FP16 cannot hold are off by 2^-25, where
the largest is 2^8 or more: 2^-33 each of the largest value in the 32 dimensions that have a reference scale in common; values that are
2^-24 of that one or less may be lost altogether.  The second sum cuts like the first, n / 16 steps of it, and parts of
it are joined a few times.  The result is rounded by half a step of its type."""
import numpy as np
import torch

from oracle import mxq_oracle as orc

import product_util as pu


def unpack(codes: np.ndarray, fmt: str) -> np.ndarray:
    return codes if orc.bits(fmt) == 8 else np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)


class Cache:
    """A cache's buffers on the host, random contents through the oracle, and their values in 64 bits."""

    def __init__(self, rng, pages, heads, dim, fmt, block, page, spread=2):
        self.fmt, self.block, self.page, self.shape = fmt, block, page, (pages, heads, page, dim)
        self.parts = []
        for _ in range(2):
            n = pages * heads * page
            x = (rng.standard_normal((n, dim)) * np.exp2(rng.integers(-spread, spread + 1, (n, 1)))).astype(np.float32)
            c, s = orc.quantize(x.reshape(-1), fmt, block)
            self.parts += [np.asarray(orc.pack(c, orc.bits(fmt))).reshape(pages, heads, page, -1).copy(),
                           np.asarray(s).reshape(pages, heads, page, -1).copy()]

    def values(self):
        kc, ks, vc, vs = self.parts
        got = []
        for c, s in ((kc, ks), (vc, vs)):
            c = unpack(c, self.fmt).astype(np.int64)
            v = pu.values64(c, s, self.fmt, self.block)
            if self.fmt == "e4m3":
                v[c & 127 == 127] = np.nan                   # S.1111.111
            got.append(v)
        return got

    def cuda(self):
        return [torch.from_numpy(p.copy()).cuda() for p in self.parts]


def tables(rng, lengths, page, pages, width=None):
    need = [-(-n // page) for n in lengths]
    width = max(1, *need) if width is None else width
    order = rng.permutation(pages)[:sum(need)]
    table = np.full((len(lengths), width), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def starts_of(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


def rows_of(values, table, n, page):
    """[n, heads, dim] of a sequence's first n tokens; where the table has no page: None in `there`."""
    t = np.arange(n)
    pages = table[t // page] if n else np.zeros(0, np.int64)
    there = (pages >= 0) & (pages < values.shape[0])
    return values[np.where(there, pages, 0), :, t % page], there


def many(dtype, dim, tokens, batch, group):
    """Whether a call is one of many queries: BF16, heads of up to 128, more than 16 rows of a cache head per sequence in the mean."""
    return dtype == torch.bfloat16 and dim <= 128 and -(-tokens // batch) * group > 16


def attention64(q, cache, table, lengths, starts, scale, causal=True, window=0, dtype=torch.bfloat16):
    """(out, lse, bound, touched) in 64 bits for q [tokens, q_heads, dim]."""
    k64, v64 = cache.values()
    tokens, q_heads, dim = q.shape
    heads = k64.shape[1]
    out, bound, lse = np.zeros(q.shape), np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    touched = np.zeros(tokens, bool)
    held = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21
    if many(dtype, dim, tokens, len(lengths), q_heads // heads):
        held = 2.0 ** -8
    entry = 0.0 if dtype == torch.bfloat16 else 2.0 ** -21
    for b, length in enumerate(lengths):
        first, n = (b, 1) if starts is None else (starts[b], starts[b + 1] - starts[b])
        touched[first:first + n] = True
        kk, there = rows_of(k64, table[b], length, cache.page)
        vv, _ = rows_of(v64, table[b], length, cache.page)
        t = np.arange(length)
        for i in range(n):
            pos = length - n + i
            seen = there & (t <= pos if causal else True)
            if window:
                seen &= t > pos - window
            if not seen.any():
                continue
            for j in range(q_heads):
                x, K, V = q[first + i, j], kk[seen, j // (q_heads // heads)], vv[seen, j // (q_heads // heads)]
                with np.errstate(invalid="ignore"):
                    s = scale * (K @ x)
                    off = abs(scale) * (np.abs(K) @ np.abs(x)) * ((dim / 16 + 16) * 2.0 ** -19 + entry)
                    p = np.exp(s - s.max())
                    lse[first + i, j] = s.max() + np.log(p.sum())
                    p /= p.sum()
                    out[first + i, j] = p @ V
                    a = np.abs(V)
                    top = np.repeat(np.where(np.isnan(a), 0, a).max(0).reshape(-1, 32).max(1), 32)
                    bound[first + i, j] = (p * (off + off.max() + 2.0 ** -20 + held)) @ a + (length / 16 + 64) * 2.0 ** -19 * (p @ a) \
                        + (length * 2.0 ** -33 + 2.0 ** -24) * top
    return out, lse, bound, touched
