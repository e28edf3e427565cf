"""What can go wrong around the operators over a paged cache of codes: NaN where it is hidden and where it is seen, pages that
are missing, extreme scales, strides, streams, captured graphs, rows that belong to nobody, a step as a server runs it."""
import math

import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq

import cache_util as cu
import product_util as pu
from oracle import mxq_oracle as orc
from test_gpu_cache import BF16, F32, FMTS, attend, ints, plain, written

pytestmark = pytest.mark.gpu

#: (queries per sequence, lengths): one, a few and many rows of a cache head, so that every kernel is met
SHAPES = [(None, [70, 129, 16]), ([3, 5], [100, 37]), ([40, 150], [333, 150])]


def poisoned(cache, table, b, pos, what, fmt, kind, block_of=0):
    """Puts a NaN into a token of a host cache: a poisoned block (every format) or a NaN code (E4M3)."""
    at = (table[b, pos // cache.page], slice(None), pos % cache.page)
    if what == "block":
        cache.parts[kind + 1][at + (block_of,)] = 255
        if kind == 0 or fmt in ("int8", "int4"):
            cache.parts[kind][at] = 0
    else:
        cache.parts[kind][at + (5,)] = 0x7F


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("counts,lengths", SHAPES)
def test_nan_reaches_those_who_see_it(fmt, dtype, dim, counts, lengths):
    for what in ("block", "code") if fmt == "e4m3" else ("block",):
        for kind in (0, 2):
            rng = np.random.default_rng(dim)
            cache = cu.Cache(rng, 40, 2, dim, fmt, 32, 16)
            table = cu.tables(rng, lengths, 16, 40)
            poisoned(cache, table, 0, lengths[0] - 2, what, fmt, kind, block_of=1)     # some queries of a sequence see it, with a window none does
            poisoned(cache, table, 1, 3, what, fmt, kind)
            for causal, window in ((True, 0), (True, 2), (False, 0)):
                got = attend(rng, cache, lengths, counts, 2, dtype, table=table, causal=causal, window=window)
                assert causal or kind or torch.isnan(got).any()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("counts,lengths", SHAPES)
def test_what_lies_behind_a_sequence_has_no_influence(fmt, counts, lengths):
    rng = np.random.default_rng(3)
    cache = cu.Cache(rng, 40, 2, 128, fmt, 32, 64)
    table = cu.tables(rng, lengths, 64, 40)
    clean = attend(rng, cache, lengths, counts, 3, BF16, table=table, q=None)
    rng = np.random.default_rng(3)
    cache = cu.Cache(rng, 40, 2, 128, fmt, 32, 64)
    table = cu.tables(rng, lengths, 64, 40)
    used = set()
    for b, n in enumerate(lengths):
        for pos in range(n):
            used.add((table[b, pos // 64], pos % 64))
    for page in range(40):
        for off in range(64):
            if (page, off) not in used:
                for kind in (0, 2):
                    cache.parts[kind][page, :, off] = 0x7F if fmt == "e4m3" else 0x77
                    cache.parts[kind + 1][page, :, off] = 255
    assert torch.equal(clean, attend(rng, cache, lengths, counts, 3, BF16, table=table, q=None))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", ["e2m1", "int8"])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("counts,lengths", SHAPES)
def test_missing_pages_are_left_out(fmt, dtype, page, counts, lengths):
    rng = np.random.default_rng(4)
    cache = cu.Cache(rng, 40, 2, 128, fmt, 32, page)
    table = cu.tables(rng, lengths, page, 40)
    table[0, 0], table[1, -(-lengths[1] // page) - 1] = -1, 40
    attend(rng, cache, lengths, counts, 2, dtype, table=table)
    table[0, :] = 1 << 30                                    # a sequence without any page sees nothing
    attend(rng, cache, lengths, counts, 2, dtype, table=table)
    bufs = cache.cuda()
    starts = cu.starts_of(lengths)
    k, v = mxq.cache_read(*bufs, ints(table), ints(starts), int(starts[-1]), fmt)
    assert not k[:lengths[0]].any() and not v[:lengths[0]].any()
    assert bool(k[lengths[0]:].any()) == (len(lengths) > 2 or lengths[1] > page)         # (of the second one the last page is missing)
    rows = plain(rng, (len(lengths), 2, 128), BF16)
    before = [t.clone() for t in bufs]
    mxq.cache_write(rows, rows, *bufs, ints(table[:, :0]), ints(lengths), fmt)          # no pages at all
    mxq.cache_write(rows[:1], rows[:1], *bufs, ints(table[:1]), ints(lengths[:1]), fmt)
    assert all(torch.equal(a, b) for a, b in zip(bufs, before))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("counts,lengths", SHAPES)
def test_values_of_very_different_sizes(fmt, dtype, counts, lengths):
    """Blocks of values from 2^-20 to 2^20, in every order: the reference that the sums are relative to has to follow."""
    for order in (1, -1):
        rng = np.random.default_rng(6)
        cache = cu.Cache(rng, 40, 2, 128, fmt, 32, 16)
        table = cu.tables(rng, lengths, 16, 40)
        for b, n in enumerate(lengths):
            for pos in range(n):
                up = int(40 * pos / n) - 20
                cache.parts[3][table[b, pos // 16], :, pos % 16] += np.uint8(order * up & 255)
        attend(rng, cache, lengths, counts, 2, dtype, table=table)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,lengths", SHAPES)
def test_scores_of_very_different_sizes(dtype, counts, lengths):
    """Scores that rise and fall by thousands along a sequence, and scales of zero and below."""
    rng = np.random.default_rng(7)
    cache = cu.Cache(rng, 40, 2, 64, "int8", 32, 16, spread=5)
    table = cu.tables(rng, lengths, 16, 40)
    for scale in (0.0, -0.2, 3.0):
        attend(rng, cache, lengths, counts, 2, dtype, table=table, scale=scale)


def test_queries_that_are_nan_or_zero():
    rng = np.random.default_rng(9)
    cache = cu.Cache(rng, 12, 1, 128, "e2m1", 32, 64)
    for dtype in (BF16, F32):
        for counts, lengths in (([1, 1, 1], [50, 60, 70]), ([60, 60, 60], [64, 70, 128])):
            q = plain(rng, (sum(counts), 2, 128), dtype)
            first = cu.starts_of(counts)
            q[first[0], 0, 7], q[first[1], 1, 0], q[first[2]] = float("nan"), float("-inf"), 0.0
            table = cu.tables(rng, lengths, 64, 12)
            out = mxq.cache_attention(q, *cache.cuda(), ints(table), ints(lengths), "e2m1", starts=ints(first))
            bad = torch.isnan(out).all(-1)
            assert bad[first[0], 0] and bad[first[1], 1] and int(bad.sum()) == 2 and int(torch.isnan(out).any(-1).sum()) == 2
            v = mxq.cache_read(*cache.cuda(), ints(table), ints(cu.starts_of(lengths)), sum(lengths), "e2m1", dtype=F32)[1]
            seen = v[sum(lengths[:2]):sum(lengths[:2]) + lengths[2] - counts[2] + 1, 0]
            assert torch.allclose(out[first[2], 0].float(), seen.mean(0), atol=0.02)       # equal weights


def test_rows_of_nobody_are_left_alone():
    rng = np.random.default_rng(11)
    cache = cu.Cache(rng, 9, 2, 64, "int4", 64, 32)
    lengths, starts = [40, 64], np.array([2, 5, 6], np.int32)
    table = cu.tables(rng, lengths, 32, 9)
    for pad in (0, 120):                                     # few rows and many
        tokens = 9 + pad
        q = plain(rng, (tokens, 4, 64), BF16)
        out, lse = torch.full_like(q, 5.0), torch.full((tokens, 4), 5.0, device="cuda")
        mxq.cache_attention(q, *cache.cuda(), ints(table), ints(lengths), "int4", block=64, starts=ints(starts), out=out, lse=lse)
        want, want_lse, bound, touched = cu.attention64(pu.to64(q), cache, table, lengths, starts, 0.125)
        assert touched.sum() == 4 and (out[~torch.from_numpy(touched)] == 5.0).all() and (lse[~torch.from_numpy(touched)] == 5.0).all()
        pu.check(out[touched], want[touched], bound[touched] + (2.0 ** -8 if pad else 0.0) * np.abs(want[touched]))
        bufs = cache.cuda()
        k, v = plain(rng, (tokens, 2, 64), F32), plain(rng, (tokens, 2, 64), F32)
        mxq.cache_write(k, v, *bufs, ints(table), ints(lengths), "int4", block=64, starts=ints(starts))
        for got, w in zip(bufs, written(cache, k.cpu().numpy(), v.cpu().numpy(), table, lengths, starts)):
            assert np.array_equal(got.cpu().numpy(), w)


def test_batches_and_sizes_that_are_empty():
    bufs = mxq.make_cache(4, 2, 128, "e4m3")
    none = torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    q = torch.zeros(0, 4, 128, dtype=BF16, device="cuda")
    assert mxq.cache_attention(q, *bufs, none, ints(np.zeros(0)), "e4m3").shape == (0, 4, 128)
    mxq.cache_write(q[:, :2], q[:, :2], *bufs, none, ints(np.zeros(0)), "e4m3")
    k, v = mxq.cache_read(*bufs, none, ints([0]), 0, "e4m3")
    assert k.shape == v.shape == (0, 2, 128)
    q = torch.ones(2, 4, 128, dtype=BF16, device="cuda")
    out = mxq.cache_attention(q, *bufs, ints(np.zeros((2, 0))), ints([5, 0]), "e4m3")
    assert not out.any()                                     # a table without pages
    out = mxq.cache_attention(q, *mxq.make_cache(0, 2, 128, "e4m3"), ints([[0], [0]]), ints([5, 0]), "e4m3")
    assert not out.any()                                     # a cache without pages


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_offsets_and_gradients(dtype):
    rng = np.random.default_rng(12)
    cache = cu.Cache(rng, 9, 2, 128, "e2m1", 32, 64)
    lengths = [100, 65, 1]
    table = cu.tables(rng, lengths, 64, 9)
    args = (*cache.cuda(), ints(table), ints(lengths), "e2m1")
    base = plain(rng, (3, 8, 128), dtype)
    want = mxq.cache_attention(base, *args)
    odd = torch.empty(3 * 8 * 129 + 1, dtype=dtype, device="cuda")[1:].view(3, 8, 129)[:, :, :128]       # rows of 129, an odd address
    odd.copy_(base)
    heads_first = base.transpose(0, 1).contiguous().transpose(0, 1)
    fused = torch.cat((base, base, base), 1)[:, 8:16]
    for q in (odd, heads_first, fused, base.clone().requires_grad_()):
        got = mxq.cache_attention(q, *args)
        assert torch.equal(got, want) and not got.requires_grad
    for t in (base[:, :2], odd[:, :2], heads_first[:, :2], fused[:, :2]):
        bufs = cache.cuda()
        mxq.cache_write(t, t, *bufs, ints(table), ints(lengths), "e2m1")
        host = base[:, :2].float().cpu().numpy()
        for got, w in zip(bufs, written(cache, host, host, table, lengths, None)):
            assert np.array_equal(got.cpu().numpy(), w)


def test_streams_workspaces_and_captured_graphs():
    rng = np.random.default_rng(13)
    cache = cu.Cache(rng, 200, 2, 128, "int8", 32, 64)
    lengths = [5000, 1200, 3000]
    table = cu.tables(rng, lengths, 64, 200)
    t, n = ints(table), ints(lengths)
    bufs = cache.cuda()
    q, kv = plain(rng, (3, 8, 128), BF16), plain(rng, (3, 4, 128), BF16)
    side = torch.cuda.Stream()
    want = mxq.cache_attention(q, *bufs, t, n, "int8")
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(mxq.cache_attention_workspace_bytes(3, 8, 3, table.shape[1], 64, 2, 128), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    got = mxq.cache_attention(q, *bufs, t, n, "int8", out=out, workspace=ws, stream=side)
    assert got is out
    other = mxq.cache_attention(q, *bufs, t, n, "int8", stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want) and torch.equal(other, want)
    # two graphs, each with a workspace of its own, replayed together; lengths change between replays
    graphs, outs = [], []
    for _ in range(2):
        mxq.cache_write(kv[:, :2], kv[:, 2:], *bufs, t, n, "int8")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mxq.cache_write(kv[:, :2], kv[:, 2:], *bufs, t, n, "int8")
            outs.append(mxq.cache_attention(q, *bufs, t, n, "int8"))
        graphs.append(g)
    for new in ([5000, 1200, 3000], [1, 1216, 0], [4999, 17, 64]):
        n.copy_(ints(new))
        q.copy_(plain(rng, (3, 8, 128), BF16))
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        want = mxq.cache_attention(q, *bufs, t, n, "int8")
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_many_queries_on_two_streams_at_once():
    rng = np.random.default_rng(16)
    lengths, counts = [600, 90], [200, 90]
    cache = cu.Cache(rng, 40, 2, 128, "e2m1", 32, 32)
    args = (*cache.cuda(), ints(cu.tables(rng, lengths, 32, 40)), ints(lengths), "e2m1")
    q, starts = plain(rng, (290, 8, 128), BF16), ints(cu.starts_of(counts))
    want = mxq.cache_attention(q, *args, starts=starts)
    graphs, outs = [], []
    for _ in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append([mxq.cache_attention(q, *args, starts=starts) for _ in range(3)])
        graphs.append(g)
    side = torch.cuda.Stream()
    for _ in range(3):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for out in outs[0] + outs[1]:
            assert torch.equal(out, want)
            out.zero_()
        torch.cuda.synchronize()
    assert mxq.load_library().mxq_wait_status(0) == 0


@pytest.mark.parametrize("counts,lengths", SHAPES + [(None, [9000, 4, 700])])
def test_results_do_not_depend_on_timing_or_on_what_the_workspace_held(counts, lengths):
    rng = np.random.default_rng(14)
    pages = sum(-(-n // 64) for n in lengths)
    cache = cu.Cache(rng, pages, 2, 128, "e4m3", 32, 64)
    table = cu.tables(rng, lengths, 64, pages)
    starts = None if counts is None else ints(cu.starts_of(counts))
    q = plain(rng, (len(lengths) if counts is None else sum(counts), 8, 128), BF16)
    bufs, n = cache.cuda(), ints(lengths)
    need = mxq.cache_attention_workspace_bytes(q.shape[0], 8, len(lengths), table.shape[1], 64, 2, 128)
    want = None
    for fill in (0, 255, 127):
        ws = torch.full((need + 64,), fill, dtype=torch.uint8, device="cuda")
        out = mxq.cache_attention(q, *bufs, ints(table), n, "e4m3", starts=starts, workspace=ws[:need])
        assert (ws[need:] == fill).all()
        assert want is None or torch.equal(out, want)
        want = out


@pytest.mark.parametrize("fmt", FMTS)
def test_a_server_s_steps(fmt):
    """A prompt in two pieces and four decoded tokens, two sequences: what the cache holds is what was written, and every step attends it."""
    rng = np.random.default_rng(15)
    heads, group, dim, page, total = 2, 4, 128, 16, (90, 41)
    bufs = mxq.make_cache(12, heads, dim, fmt, page=page)
    table = cu.tables(rng, total, page, 12)
    k = [plain(rng, (n, heads, dim), BF16) for n in total]
    v = [plain(rng, (n, heads, dim), BF16) for n in total]
    host = cu.Cache(rng, 12, heads, dim, fmt, 32, page)
    for p in host.parts:
        p[:] = 0
    done = [0, 0]
    for counts in ([50, 20], [36, 17], [1, 1], [1, 1], [1, 1], [1, 1]):
        lengths = [d + c for d, c in zip(done, counts)]
        starts = cu.starts_of(counts)
        kk = torch.cat([x[d:d + c] for x, d, c in zip(k, done, counts)])
        vv = torch.cat([x[d:d + c] for x, d, c in zip(v, done, counts)])
        one = all(c == 1 for c in counts)
        mxq.cache_write(kk, vv, *bufs, ints(table), ints(lengths), fmt, starts=None if one else ints(starts))
        host.parts = written(host, kk.float().cpu().numpy(), vv.float().cpu().numpy(), table, lengths, starts)
        for got, w in zip(bufs, host.parts):
            assert np.array_equal(got.cpu().numpy(), w)
        q = plain(rng, (int(starts[-1]), heads * group, dim), BF16)
        out = mxq.cache_attention(q, *bufs, ints(table), ints(lengths), fmt, starts=None if one else ints(starts))
        want, _, bound, _ = cu.attention64(pu.to64(q), host, table, lengths, starts, 1 / math.sqrt(dim))
        pu.check(out, want, bound)
        done = lengths
    assert mxq.load_library().mxq_wait_status(0) == 0
    ref = orc.quantize(k[0].float().cpu().numpy().reshape(-1), fmt, 32)
    read = mxq.cache_read(*bufs, ints(table[:1]), ints([0, total[0]]), total[0], fmt)[0]
    want = mxq.dequantize(torch.from_numpy(np.asarray(orc.pack(ref[0], orc.bits(fmt)))).cuda(), torch.from_numpy(np.asarray(ref[1])).cuda(),
                          k[0].numel(), fmt, dtype=BF16)
    assert torch.equal(read.reshape(-1), want)
