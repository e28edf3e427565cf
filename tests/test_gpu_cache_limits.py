"""The operators over a paged cache of codes at the limits of what their description allows: sequences as long as 32 bits count, many
sequences in a call, caches beyond 4 GB."""
import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq

import cache_util as cu
import product_util as pu
from test_gpu_cache import BF16, F32, attend, ints, plain

pytestmark = pytest.mark.gpu

LONGEST = (1 << 31) - 1                                      # tokens


def repeated(pages):
    """The table of one sequence of 2^31 tokens in `pages` pages of 256, in turn."""
    return (torch.arange(1 << 23, device="cuda", dtype=torch.int32) % pages).view(1, -1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", ["e2m1", "int8"])
@pytest.mark.parametrize("n", [1, 5, 70])
def test_the_last_tokens_of_the_longest_sequence(fmt, dtype, n):
    """Windows at the end of a sequence of 2^31 - 1 tokens: one, a few and many rows of a cache head."""
    rng = np.random.default_rng(n)
    cache = cu.Cache(rng, 3, 1, 128, fmt, 32, 256)
    q = plain(rng, (n, 2, 128), dtype)
    starts = None if n == 1 else np.array([0, n], np.int32)
    table = repeated(3)
    for window in (1, 333):
        got = mxq.cache_attention(q, *cache.cuda(), table, ints([LONGEST]), fmt, starts=None if n == 1 else ints(starts), window=window)
        last = 5 * 256 - 1                                   # the same tokens at the end of a sequence of five pages
        want, _, bound, _ = cu.attention64(pu.to64(q), cache, table[:, -5:].cpu().numpy(), [last], np.array([0, n], np.int32), 128 ** -0.5, True, window, dtype)
        pu.check(got, want, bound)
    if n == 1:                                               # and the newest token written and attended by itself
        bufs = cache.cuda()
        k, v = plain(rng, (1, 1, 128), dtype), plain(rng, (1, 1, 128), dtype)
        mxq.cache_write(k, v, *bufs, table, ints([LONGEST]), fmt)
        got = mxq.cache_attention(q, *bufs, table, ints([LONGEST]), fmt, window=1)
        page = int(table[0, -1])
        alone = mxq.cache_read(*bufs, ints([[page]]), ints([0, 255]), 255, fmt, dtype=dtype)[1][254]
        assert torch.equal(got[0], alone.expand(2, 128))
        before = cache.cuda()
        assert sum(int((a != b).any(-1).sum()) for a, b in zip(bufs, before)) <= 4      # one row of each buffer


def test_all_tokens_of_the_longest_sequence():
    rng = np.random.default_rng(3)
    cache = cu.Cache(rng, 3, 1, 64, "e2m1", 32, 256)
    q = plain(rng, (1, 2, 64), BF16)
    lse = torch.empty(1, 2, device="cuda")
    got = mxq.cache_attention(q, *cache.cuda(), repeated(3), ints([LONGEST]), "e2m1", lse=lse)
    k64, v64 = (x.transpose(0, 2, 1, 3).reshape(768, 64) for x in cache.values())
    times = np.full(768, LONGEST // 768)
    times[:LONGEST % 768] += 1
    s = pu.to64(q)[0] @ k64.T / 8
    p = times * np.exp(s - s.max(-1, keepdims=True))
    total = p.sum(-1, keepdims=True)
    # each lane adds up to 2^31 / (148 * 128) weights one by one: 2^17 of them, 2^-24 each
    want, mags = p / total @ v64, p / total @ np.abs(v64)
    pu.check(got, want[None], (mags * (2.0 ** -11 + 2.0 ** -6) + 2.0 ** -19)[None])
    assert np.abs(pu.to64(lse)[0] - (s.max(-1) + np.log(total[:, 0]))).max() <= 2.0 ** -6


@pytest.mark.parametrize("dtype,dim", [(F32, 64), (F32, 256), (BF16, 256), (BF16, 64)])
@pytest.mark.parametrize("group,counts,lengths", [(5, [300, 0, 7, 90], [310, 5, 7, 1000]), (3, [1] * 40 + [129], [33] * 40 + [140]), (16, [70, 1], [90, 640])])
def test_items_of_a_run_are_followed(dtype, dim, group, counts, lengths):
    """Sequences of many items, groups of heads that do not divide an item's rows, runs over several heads and sequences."""
    rng = np.random.default_rng(group)
    cache = cu.Cache(rng, sum(-(-n // 32) for n in lengths) + 1, 2, dim, "int8", 32, 32)
    for causal, window in ((True, 0), (True, 50), (False, 0)):
        attend(rng, cache, lengths, counts, group, dtype, causal=causal, window=window)


def test_time_grows_like_the_queries():
    """FP32 queries with a window: four times as many take four times as long (sixteen times, where each item is searched for)."""
    rng = np.random.default_rng(2)
    cache = cu.Cache(rng, 2, 1, 64, "int8", 32, 256).cuda()
    took = []
    for n in (8192, 32768):
        q, table = plain(rng, (n, 16, 64), F32), repeated(2)[:, :n // 256].contiguous()
        args = (q, *cache, table, ints([n]), "int8")
        mxq.cache_attention(*args, starts=ints([0, n]), window=64)
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            mxq.cache_attention(*args, starts=ints([0, n]), window=64)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        took.append(sorted(times)[2])
    print("%.3f and %.3f ms" % tuple(took))
    assert took[1] <= 8 * took[0]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group", [1, 8])
@pytest.mark.parametrize("counts,lengths", [([8], [5]), ([40, 3], [5, 40]), ([1, 2], [0, 1])])
def test_a_window_without_limit(dtype, group, counts, lengths):
    """Windows up to what their type holds, also where sequences bring more queries than they have tokens."""
    rng = np.random.default_rng(4)
    cache = cu.Cache(rng, 6, 1, 64, "int8", 32, 16)
    table = cu.tables(rng, lengths, 16, 6)
    q = plain(rng, (sum(counts), group, 64), dtype)
    want = attend(rng, cache, lengths, counts, group, dtype, table=table, q=q)
    for window in (64, 1 << 30, (1 << 31) - 64, (1 << 31) - 1, 1 << 31, 1 << 40, (1 << 62) + 5):
        got = mxq.cache_attention(q, *cache.cuda(), ints(table), ints(lengths), "int8", starts=ints(cu.starts_of(counts)), window=window)
        assert torch.equal(got, want), window


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("batch,n,group,dim", [(300, 1, 2, 64), (1100, 1, 1, 128), (200, 2, 3, 256), (600, 3, 8, 64)])
def test_more_sequences_than_threads(dtype, batch, n, group, dim):
    """A CTA plans several sequences per thread; some of them are empty, some have no tokens that are new."""
    rng = np.random.default_rng(batch)
    lengths = [int(x) for x in rng.integers(0, 60, batch)]
    counts = [n if n == 1 or b % 7 else 0 for b in range(batch)]
    cache = cu.Cache(rng, sum(-(-x // 16) for x in lengths), 1, dim, "int8", 32, 16)
    attend(rng, cache, lengths, None if n == 1 else counts, group, dtype)
    attend(rng, cache, lengths, counts, group, dtype, window=20)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_beyond_4_gb(dtype):
    """Tokens in the last pages of a cache of 5.2 GB of codes each for keys and values: the bytes and results of a small cache."""
    rng = np.random.default_rng(6)
    pages, page, heads, dim = 80000, 64, 8, 128
    large = mxq.make_cache(pages, heads, dim, "e4m3", page=page)
    small = mxq.make_cache(12, heads, dim, "e4m3", page=page)
    assert large[0].numel() > 1 << 32
    near = np.array([[0, 5, 11], [3, 7, 2], [10, 1, -1]], np.int32)
    far = np.where(near < 0, -1, np.where(near % 2, near * 3, pages - 1 - near)).astype(np.int32)
    lengths, counts = [190, 129, 128], [190, 129, 128]
    k, v = plain(rng, (sum(counts), heads, dim), dtype), plain(rng, (sum(counts), heads, dim), dtype)
    got = []
    for cache, table in ((small, near), (large, far)):
        starts = ints(cu.starts_of(counts))
        mxq.cache_write(k, v, *cache, ints(table), ints(lengths), "e4m3", starts=starts)
        out = [*mxq.cache_read(*cache, ints(table), starts, sum(lengths), "e4m3", dtype=dtype)]
        for n in (1, 2, 50):
            q = k[:3 * n].repeat_interleave(2, 1)
            out.append(mxq.cache_attention(q, *cache, ints(table), ints(lengths), "e4m3", starts=ints([0, n, 2 * n, 3 * n])))
        got.append(out)
    assert got[0][0].abs().max() > 1 and all(torch.equal(a, b) for a, b in zip(*got))
