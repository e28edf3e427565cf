"""The operators over a paged cache of codes against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq

import cache_util as cu
import product_util as pu
from oracle import mxq_oracle as orc

pytestmark = pytest.mark.gpu

FMTS = ["e4m3", "e2m1", "int8", "int4"]
BF16, F32 = torch.bfloat16, torch.float32


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def plain(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().to(dtype)


def attend(rng, cache, lengths, counts, group, dtype, pages_of=None, table=None, scale=None, causal=True, window=0, q=None, **kw):
    pages, heads, page, dim = cache.shape
    table = cu.tables(rng, lengths, page, pages) if table is None else table
    starts = None if counts is None else cu.starts_of(counts)
    tokens = len(lengths) if counts is None else int(starts[-1])
    q = plain(rng, (tokens, heads * group, dim), dtype) if q is None else q
    lse = torch.full((tokens, heads * group), 7.0, device="cuda")
    got = mxq.cache_attention(q, *cache.cuda(), ints(table), ints(lengths), cache.fmt, block=cache.block,
                              starts=None if starts is None else ints(starts), scale=scale, causal=causal, window=window, lse=lse, **kw)
    want, want_lse, bound, _ = cu.attention64(pu.to64(q), cache, table, lengths, starts, dim ** -0.5 if scale is None else scale, causal, window, dtype)
    pu.check(got, want, bound)
    seen = np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(want_lse), np.isneginf(pu.to64(lse)))
    top = np.abs(pu.to64(q)).max() * max(np.nanmax(np.abs(v)) for v in cache.values()) * dim * abs(dim ** -0.5 if scale is None else scale)
    assert np.abs(pu.to64(lse)[seen] - want_lse[seen]).max(initial=0.0) <= (dim / 16 + 20) * 2.0 ** -19 * max(top, 1.0)
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim,block,page", [(64, 32, 16), (64, 64, 64), (128, 32, 64), (128, 64, 32), (128, 128, 128), (256, 32, 16), (256, 128, 256)])
def test_one_query_per_sequence(fmt, dtype, dim, block, page):
    rng = np.random.default_rng(dim + block + page)
    lengths = [1, 0, 15, 16, 17, 63, 64, 65, 300]
    cache = cu.Cache(rng, sum(-(-n // page) for n in lengths) + 2, 2, dim, fmt, block, page)
    attend(rng, cache, lengths, None, 4, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16, 33])
def test_groups_of_heads(fmt, dtype, group):
    rng = np.random.default_rng(group)
    cache = cu.Cache(rng, 12, 3, 64, fmt, 32, 32)
    attend(rng, cache, [100, 33, 130], None, group, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("counts,lengths", [([3, 1, 0, 5], [70, 1, 40, 5]), ([40, 7], [150, 7]), ([6, 2], [4, 0])])
def test_several_queries(fmt, dtype, dim, counts, lengths):
    rng = np.random.default_rng(sum(counts) + dim)
    cache = cu.Cache(rng, 20, 2, dim, fmt, 32, 16)
    for causal, window in ((True, 0), (True, 9), (True, 1), (False, 0)):
        attend(rng, cache, lengths, counts, 3, dtype, causal=causal, window=window)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim,block,page,group,counts,lengths", [
    (128, 32, 64, 1, [130], [130]), (128, 64, 16, 2, [70, 200, 0, 129], [500, 200, 9, 140]), (64, 32, 32, 4, [300, 33], [301, 640]),
    (128, 128, 128, 8, [33, 1], [1000, 3]), (64, 64, 256, 3, [90, 90], [60, 777])])
def test_many_queries(fmt, dim, block, page, group, counts, lengths):
    rng = np.random.default_rng(sum(counts))
    cache = cu.Cache(rng, sum(-(-n // page) for n in lengths) + 1, 2, dim, fmt, block, page)
    for causal, window in ((True, 0), (True, 100), (False, 0)):
        attend(rng, cache, lengths, counts, group, BF16, causal=causal, window=window)


@pytest.mark.parametrize("fmt,dtype", [("e2m1", BF16), ("int4", F32), ("e4m3", BF16), ("int8", F32)])
def test_long_contexts_in_parts(fmt, dtype):
    rng = np.random.default_rng(5)
    cache = cu.Cache(rng, 80, 2, 128, fmt, 32, 128)
    attend(rng, cache, [9001], None, 4, dtype)
    attend(rng, cache, [5000, 3, 777, 2049], None, 2, dtype, window=2000)
    attend(rng, cache, [6000, 900], [2, 1], 4, dtype)


# ---- writing and reading ------------------------------------------------------------------------------------------


def written(cache, k, v, table, lengths, starts):
    """The host cache's parts after the tokens' rows are written, through the oracle."""
    parts = [p.copy() for p in cache.parts]
    pages, heads, page, dim = cache.shape
    for b, length in enumerate(lengths):
        first, n = (b, 1) if starts is None else (starts[b], starts[b + 1] - starts[b])
        for i in range(n):
            pos = length - n + i
            if pos < 0 or not 0 <= table[b, pos // page] < pages:
                continue
            for at, x in ((0, k), (2, v)):
                c, s = orc.quantize(np.ascontiguousarray(x[first + i]).reshape(-1), cache.fmt, cache.block)
                parts[at][table[b, pos // page], :, pos % page] = np.asarray(orc.pack(c, orc.bits(cache.fmt))).reshape(heads, -1)
                parts[at + 1][table[b, pos // page], :, pos % page] = np.asarray(s).reshape(heads, -1)
    return parts


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads,dim,block,page", [(1, 64, 32, 16), (3, 64, 64, 64), (8, 128, 32, 64), (5, 128, 128, 32), (2, 256, 64, 256)])
def test_write_then_read(fmt, dtype, heads, dim, block, page):
    rng = np.random.default_rng(heads + dim)
    lengths, counts = [page, 1, 0, 2 * page + 3, 40], [page, 1, 0, 7, 2]
    cache = cu.Cache(rng, 24, heads, dim, fmt, block, page)
    table, starts = cu.tables(rng, lengths, page, 24), cu.starts_of(counts)
    tokens = int(starts[-1])
    kv = plain(rng, (tokens, heads, 3, dim), dtype)                     # strided slices
    kv[0, 0, 0, 0], kv[-1, -1, 1, 5], kv[0, 0, 1] = float("nan"), float("inf"), 0.0
    k, v = kv[:, :, 0], kv[:, :, 1]
    bufs = cache.cuda()
    mxq.cache_write(k, v, *bufs, ints(table), ints(lengths), fmt, block=block, starts=ints(starts))
    want = written(cache, k.float().cpu().numpy(), v.float().cpu().numpy(), table, lengths, starts)
    for got, w in zip(bufs, want):
        assert np.array_equal(got.cpu().numpy(), w)
    firsts = cu.starts_of(lengths)
    out = tuple(torch.full((int(firsts[-1]) + 2, heads, dim), 3.0, dtype=dtype, device="cuda") for _ in range(2))
    mxq.cache_read(*bufs, ints(table), ints(firsts), int(firsts[-1]) + 2, fmt, block=block, out=out)
    for o, codes, scales in ((out[0], *want[:2]), (out[1], *want[2:])):
        ref = mxq.dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 24 * heads * page * dim, fmt, block, dtype)
        ref = ref.view(24, heads, page, dim)
        rows = torch.cat([ref[torch.from_numpy(table[b].astype(np.int64)).cuda()[torch.arange(n, device="cuda") // page], :,
                              torch.arange(n, device="cuda") % page] for b, n in enumerate(lengths) if n])
        assert torch.equal(o[:-2].view(torch.int16 if dtype == BF16 else torch.int32), rows.view(torch.int16 if dtype == BF16 else torch.int32))
        assert (o[-2:] == 3.0).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_one_token_per_sequence_and_a_padded_slot(fmt):
    rng = np.random.default_rng(8)
    lengths = [17, 0, 1, 64]
    cache = cu.Cache(rng, 9, 4, 128, fmt, 32, 16)
    table = cu.tables(rng, lengths, 16, 9)
    k, v = plain(rng, (4, 4, 128), BF16), plain(rng, (4, 4, 128), BF16)
    bufs = cache.cuda()
    mxq.cache_write(k, v, *bufs, ints(table), ints(lengths), fmt)
    for got, w in zip(bufs, written(cache, k.float().cpu().numpy(), v.float().cpu().numpy(), table, lengths, None)):
        assert np.array_equal(got.cpu().numpy(), w)
