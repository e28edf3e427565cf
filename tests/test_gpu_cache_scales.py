"""Values and scores of very different sizes in cache_attention: what a row does not see has no influence on it however large it is, and what it
sees counts by its weight.

Bounds.  As in cache_util, but for what FP16 cannot hold.  A row's weights times the values' scales are FP16 numbers relative to the largest
such product of the row and the block, or to a scale of which the largest weight's own is 2^-5 (FP32 queries; BF16: 2^-8) or more while that
weight counts 2^7 or more: each is off by 2^-25 (1 + 2^3) where the largest product is 2^2 (2^-1) or more, less than 2^-23 (2^-20) of it, counted
by the blocks' scales and the largest element of the format.  Weights are FP32 numbers relative to a maximum that is at most 2^12 below the scores of those who share it
and 2^8 or more below the row's largest, and numbers below 2^-126 become zeros there: a weight below 2^-120 may not count.  With many queries a
weight is rounded to BF16, by 2^-8 of it, and divided by a sum of rounded ones, which is off by 2^-8 too: 2^-7 together."""
import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq

import cache_util as cu
import product_util as pu
from test_gpu_cache import BF16, F32, FMTS, ints, plain

pytestmark = pytest.mark.gpu

MOST = {"e4m3": 448.0, "e2m1": 6.0, "int8": 128.0, "int4": 8.0}


def check(q, cache, lengths, counts, table, dtype, scale=None, causal=True, window=0, rows=None):
    """The call's results against 64 bits, within bounds that weigh what is lost by the softmax's weights; `rows`: those that are looked at."""
    heads, dim = cache.shape[1], cache.shape[3]
    group, starts = q.shape[1] // heads, cu.starts_of([1] * len(lengths) if counts is None else counts)
    scale = dim ** -0.5 if scale is None else scale
    lse = torch.empty(q.shape[:2], device="cuda")
    got = mxq.cache_attention(q, *cache.cuda(), ints(table), ints(lengths), cache.fmt, block=cache.block, starts=None if counts is None else ints(starts),
                              scale=scale, causal=causal, window=window, lse=lse)
    k64, v64 = cache.values()
    vs = np.repeat(pu.scale64(cache.parts[3]), cache.block, -1)[..., ::32] * MOST[cache.fmt]        # per 32 dimensions
    q64, many = pu.to64(q), cu.many(dtype, dim, q.shape[0], len(lengths), group)
    want, bound = np.zeros(q.shape), np.zeros(q.shape)
    held = 2.0 ** -7 if many else 2.0 ** -11 if dtype == BF16 else 2.0 ** -21
    for b, length in enumerate(lengths):
        kk, there = cu.rows_of(k64, table[b], length, cache.page)
        vv, ss = (cu.rows_of(x, table[b], length, cache.page)[0] for x in (v64, vs))
        t = np.arange(length)
        for i in range(starts[b + 1] - starts[b]):
            pos = length - (starts[b + 1] - starts[b]) + i
            seen = there & (t <= pos if causal else True) & (t > pos - window if window else True)
            if not seen.any():
                continue
            for j in range(q.shape[1]):
                x, K, V, S = q64[starts[b] + i, j], kk[seen, j // group], vv[seen, j // group], ss[seen, j // group]
                s = scale * (K @ x)
                off = abs(scale) * (np.abs(K) @ np.abs(x)) * ((dim / 16 + 16) * 2.0 ** -19 + (0.0 if dtype == BF16 else 2.0 ** -21))
                p = np.exp(s - s.max())
                p /= p.sum()
                top = np.repeat((p[:, None] * S).max(0), 32)
                want[starts[b] + i, j] = p @ V
                bound[starts[b] + i, j] = (p * (np.expm1(off + p @ off) + 2.0 ** -20 + held)) @ np.abs(V) \
                    + (length / 16 + 64) * 2.0 ** -19 * (p @ np.abs(V)) + length * 2.0 ** (-20 if dtype == BF16 else -23) * top + np.where(p < 2.0 ** -120, p, 0) @ np.abs(V)
    rows = slice(None) if rows is None else rows
    pu.check(got[rows], want[rows], bound[rows])
    return got, lse


def grow(cache, table, b, pos, by):
    """The values of a token times 2^by."""
    at = (table[b, pos // cache.page], slice(None), pos % cache.page)
    s = cache.parts[3][at].astype(np.int64) + by
    cache.parts[3][at] = np.clip(s, 1, 254).astype(np.uint8)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("by", [9, 30, 100, -30, -100])
@pytest.mark.parametrize("counts,lengths,at", [([2], [3], 2), ([2], [200], 199), ([5], [100], 97), ([5, 2], [40, 100], 36), ([7], [700], 3), ([60], [130], 100)])
def test_hidden_values_of_another_size(fmt, dtype, by, counts, lengths, at):
    """One token far above or below the others, which some of a sequence's queries see and others do not, behind them or out of their window."""
    for dim, group in ((64, 1), (128, 3), (256, 2)):
        rng = np.random.default_rng(dim)
        cache = cu.Cache(rng, 60, 2, dim, fmt, 32, 16)
        table = cu.tables(rng, lengths, 16, 60)
        grow(cache, table, 0, at, by)
        q = plain(rng, (sum(counts), 2 * group, dim), dtype)
        for window in (0, 3, lengths[0] - at):
            check(q, cache, lengths, counts, table, dtype, window=window)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("length,at", [(40, 0), (40, 20), (700, 650), (700, 1), (5000, 2500)])
def test_a_loud_value_of_a_small_weight(fmt, dtype, length, at):
    """A token whose value is 2^up times the others', with a weight of about 2^-92: for up = 30 and 60 it does not count, for 92 as much as the
    others, for 110 it is all there is."""
    rng = np.random.default_rng(at)
    for dim in (64, 128):
        for up in (30, 60, 92, 110):
            cache = cu.Cache(rng, -(-length // 64), 1, dim, fmt, 32, 64, spread=0)
            table = cu.tables(rng, [length], 64, -(-length // 64))
            grow(cache, table, 0, at, up)
            place = (table[0, at // 64], slice(None), at % 64)
            one = {"e4m3": 0xB8, "e2m1": 0xAA, "int8": 0x81, "int4": 0x99}[fmt]         # -1, -1, -127, -7
            cache.parts[0][place], cache.parts[1][place] = one, {"e4m3": 127, "e2m1": 127, "int8": 120, "int4": 124}[fmt]
            value = {"e4m3": 1, "e2m1": 1, "int8": 127 / 128, "int4": 7 / 8}[fmt]
            q = torch.full((1, 2, dim), 0.01, device="cuda", dtype=dtype)
            q[:, :, :2] = 64 / (2 * value)                   # scores: -64 for the token, a small normal number times 32 for the others
            keep = cache.parts[0][place].copy()
            cache.parts[0][..., :2 if fmt in ("e4m3", "int8") else 1] = 0        # the others' first two elements: 0
            cache.parts[0][place] = keep
            check(q, cache, [length], None, table, dtype, scale=1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("counts,lengths", [(None, [70, 129, 16]), ([3, 5], [100, 37]), ([40, 150], [333, 150])])
def test_values_of_every_size(fmt, dtype, counts, lengths):
    """Each token's blocks at a scale of their own, over nearly the whole range; scores flat and steep."""
    for dim, block in ((64, 32), (128, 64), (256, 128)):
        rng = np.random.default_rng(dim)
        cache = cu.Cache(rng, 40, 2, dim, fmt, block, 16)
        table = cu.tables(rng, lengths, 16, 40)
        cache.parts[3] = rng.integers(1, 200, cache.parts[3].shape).astype(np.uint8)
        q = plain(rng, (sum(counts or [1] * len(lengths)), 4, dim), dtype)
        for scale, window in ((0.1, 0), (4.0, 0), (0.1, 7)):
            check(q, cache, lengths, counts, table, dtype, scale=scale, window=window)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", ["e2m1", "int8"])
def test_a_small_first_token_and_blocks_of_zeros(fmt, dtype):
    rng = np.random.default_rng(1)
    lengths = [900, 77, 1]
    cache = cu.Cache(rng, 40, 2, 128, fmt, 32, 64)
    table = cu.tables(rng, lengths, 64, 40)
    for b in range(3):
        grow(cache, table, b, 0, -12)
    for pos in (5, 6, 76, 300):
        at = (table[0, pos // 64], slice(None), pos % 64)
        cache.parts[2][at], cache.parts[3][at] = 0, 0
    cache.parts[2][table[1, 0]], cache.parts[3][table[1, 0], ..., 1] = 0, 0
    check(plain(rng, (3, 8, 128), dtype), cache, lengths, None, table, dtype)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("byte", [245, 248, 250, 253, 254])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("counts,lengths,at,group", [([60], [130], 100, 1), ([140, 33], [140, 200], 139, 2), ([3], [90], 89, 2)])
def test_hidden_values_beyond_the_type(fmt, byte, dim, counts, lengths, at, group):
    """The largest elements under the largest scales, which BF16 cannot hold, behind a query or out of its window."""
    rng = np.random.default_rng(dim)
    cache = cu.Cache(rng, 30, 2, dim, fmt, 32, 16)
    table = cu.tables(rng, lengths, 16, 30)
    place = (table[0, at // 16], slice(None), at % 16)
    cache.parts[2][place], cache.parts[3][place] = {"e4m3": 0x7E, "e2m1": 0x7F, "int8": 0x81, "int4": 0x97}[fmt], byte
    q = plain(rng, (sum(counts), 2 * group, dim), BF16)
    for window in (0, 5):
        pos = lengths[0] - counts[0] + np.arange(counts[0])
        hidden = (pos < at) | ((pos >= at + window) if window else False)
        rows = torch.from_numpy(np.concatenate((np.flatnonzero(hidden), np.arange(counts[0], sum(counts)))))
        check(q, cache, lengths, counts, table, BF16, window=window, rows=rows)


@pytest.mark.parametrize("fmt", FMTS)
def test_many_queries_over_small_values(fmt):
    rng = np.random.default_rng(5)
    cache = cu.Cache(rng, 30, 2, 128, fmt, 32, 16, spread=0)
    table = cu.tables(rng, [130], 16, 30)
    for down in (0, 60, 100):
        parts = cache.parts[3].copy()
        cache.parts[3] = (cache.parts[3] - down).astype(np.uint8)
        check(plain(rng, (60, 2, 128), BF16), cache, [130], [60], table, BF16)
        cache.parts[3] = parts


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("counts,lengths", [(None, [70, 129, 1]), ([3, 5], [100, 37]), ([40, 150], [333, 150]), (None, [9000])])
@pytest.mark.parametrize("scale", [2.0 ** 24, -2.0 ** 28, 2.0 ** 30, 2.0 ** 40, -2.0 ** 70, 1e30, -1e31, 3e35, -3e35])
def test_scores_of_every_finite_size(fmt, dtype, counts, lengths, scale):
    """Keys that are all alike weigh alike, however large their scores are; the logarithm of the sum is the score's."""
    rng = np.random.default_rng(3)
    cache = cu.Cache(rng, 150, 2, 64, fmt, 32, 64)
    table = cu.tables(rng, lengths, 64, 150)
    one = {"e4m3": (0x3A, 127), "e2m1": (0x33, 127), "int8": (0x5B, 121), "int4": (0x55, 125)}[fmt]       # 1.25, 1.5, 91 / 64, 5 / 4
    cache.parts[0][:], cache.parts[1][:] = one
    q = torch.empty(sum(counts or [1] * len(lengths)), 4, 64, device="cuda").uniform_(0.5, 1.0, generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
    starts = cu.starts_of([1] * len(lengths) if counts is None else counts)
    lse = torch.empty(q.shape[:2], device="cuda")
    got = mxq.cache_attention(q, *cache.cuda(), ints(table), ints(lengths), fmt, starts=None if counts is None else ints(starts), scale=scale, lse=lse)
    k64, v64 = cache.values()
    s = scale * (pu.to64(q) @ k64[0, 0, 0])
    assert np.isfinite(s.astype(np.float32)).all()
    g = pu.to64(got)
    assert np.isfinite(g).all()
    # a score is off by 2^-17 of itself; weights that are alike are rounded alike
    assert (np.abs(pu.to64(lse) - s) <= 2.0 ** -17 * np.abs(s) + 16).all()
    for b, n in enumerate(starts[1:] - starts[:-1]):
        V = cu.rows_of(v64, table[b], lengths[b], 64)[0]
        for i in range(n):
            seen = V[:lengths[b] - n + i + 1]
            for j in range(4):
                want, a = seen[:, j // 2].mean(0), np.abs(seen[:, j // 2]).mean(0)
                # weights: 8, 11 or 22 bits, each the same; sums: as everywhere
                assert (np.abs(g[starts[b] + i, j] - want) <= (2.0 ** -7 + (lengths[b] / 16 + 64) * 2.0 ** -19) * a + pu.half_step(dtype) * np.abs(want)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("counts,lengths", [(None, [70, 129, 16]), ([3, 5], [100, 37]), ([60, 110], [333, 150])])
def test_nan_among_values_of_every_size(fmt, dtype, counts, lengths):
    """Poisoned blocks and NaN codes, seen by some rows and hidden from others, where scales lie far apart."""
    for kind in (0, 2):
        rng = np.random.default_rng(8)
        cache = cu.Cache(rng, 40, 2, 128, fmt, 32, 16)
        table = cu.tables(rng, lengths, 16, 40)
        cache.parts[3] = rng.integers(60, 180, cache.parts[3].shape).astype(np.uint8)
        for b, pos in ((0, lengths[0] - 2), (1, 3)):
            at = (table[b, pos // 16], slice(None), pos % 16)
            cache.parts[kind + 1][at + (1,)] = 255
            if fmt == "e4m3":
                cache.parts[kind][at + (5,)] = 0x7F
        q = plain(rng, (sum(counts or [1] * len(lengths)), 4, 128), dtype)
        for causal, window in ((True, 0), (True, 2), (False, 0)):
            check(q, cache, lengths, counts, table, dtype, scale=0.1, causal=causal, window=window)
