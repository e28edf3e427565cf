"""The operators over a paged cache in the bounds-checked build: sizes where index arithmetic goes wrong first, with exactly sized
buffers; every plain and asynchronous access of the kernels lies in the buffers that the call was given."""
import ctypes
import os

import pytest
import torch

from paper_2604_00529_b200.binding import FORMATS, _Batch, _Cache, _Rows

from test_debug_build import LIB, Info, P, report, u8
from test_debug_products import clean, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    if not os.path.exists(LIB):
        pytest.fail("libmxq_debug.so is not built: python -m paper_2604_00529_b200.build --debug")
    L = ctypes.CDLL(LIB)
    vp, sz, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    c, b, r = ctypes.POINTER(_Cache), ctypes.POINTER(_Batch), ctypes.POINTER(_Rows)
    L.mxq_cache_write.argtypes = [c, b, r, r, i, sz, vp]
    L.mxq_cache_read.argtypes = [c, b, sz, vp, vp, i, vp]
    L.mxq_cache_attention_workspace_bytes.argtypes = [c, b, i, i, sz]
    L.mxq_cache_attention_workspace_bytes.restype = sz
    L.mxq_cache_attention.argtypes = [c, b, r, i, i, sz, ctypes.c_float, i, sz, vp, vp, vp, sz, vp]
    L.mxq_debug_report.argtypes = [ctypes.POINTER(Info), i]
    return L


@pytest.mark.parametrize("fmt,bits", [("e4m3", 8), ("e2m1", 4), ("int8", 8), ("int4", 4)])
@pytest.mark.parametrize("counts,lengths,page,dim,block,heads,group", [
    ([1, 1, 1], [1, 16, 17], 16, 64, 64, 1, 1), ([1], [3000], 64, 128, 32, 2, 4), ([1] * 90, [130] * 90, 32, 128, 128, 2, 3),
    ([2, 0, 9], [40, 7, 9], 16, 256, 32, 3, 5), ([70, 1], [200, 64], 64, 64, 32, 2, 4), ([130], [140], 128, 128, 64, 1, 2)])
def test_cache_stays_inside(D, counts, lengths, page, dim, block, heads, group, fmt, bits):
    stream = torch.cuda.current_stream().cuda_stream
    need = [-(-n // page) for n in lengths]
    pages, width, batch, tokens = sum(need), max(need), len(counts), sum(counts)
    n = pages * heads * page * dim
    kc, ks, vc, vs = some(n * bits // 8), some(n // block), some(n * bits // 8), some(n // block)
    table, at = torch.full((batch, width), -1, dtype=torch.int32), 0
    for b, m in enumerate(need):
        table[b, :m] = torch.arange(at, at + m)
        at += m
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    table, starts, first = table.cuda(), ints([sum(counts[:b]) for b in range(batch + 1)]), ints([sum(lengths[:b]) for b in range(batch + 1)])
    lengths_d = ints(lengths)
    cache = _Cache(P(kc), P(ks), P(vc), P(vs), pages, page, heads, dim, FORMATS[fmt], block)
    for dtype, size in ((0, 4), (1, 2)):
        for given in ((starts, None) if set(counts) == {1} else (starts,)):
            report(D)
            b = _Batch(P(table), P(lengths_d), None if given is None else P(given), batch, width)
            q_heads = heads * group
            q, out, lse = some(tokens * q_heads * dim * size), u8(tokens * q_heads * dim * size), u8(tokens * q_heads * 4)
            rows, kv = _Rows(P(q), q_heads * dim, dim), some(tokens * heads * dim * size)
            kr = _Rows(P(kv), heads * dim, dim)
            assert D.mxq_cache_write(ctypes.byref(cache), ctypes.byref(b), ctypes.byref(kr), ctypes.byref(kr), dtype, tokens, stream) == 0
            ws_bytes = D.mxq_cache_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(b), q_heads, dtype, tokens)
            ws = u8(ws_bytes)
            assert D.mxq_cache_attention(ctypes.byref(cache), ctypes.byref(b), ctypes.byref(rows), q_heads, dtype, tokens, 0.1, 1, 0, P(out), P(lse),
                                         P(ws), ws_bytes, stream) == 0
            total = sum(lengths)
            k, v = u8(total * heads * dim * size), u8(total * heads * dim * size)
            rb = _Batch(P(table), None, P(first), batch, width)
            assert D.mxq_cache_read(ctypes.byref(cache), ctypes.byref(rb), total, P(k), P(v), dtype, stream) == 0
            clean(D, 3)
