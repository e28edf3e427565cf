"""The operators over a paged cache in the bounds-checked build, beyond single calls of plain batches: windows, items in parts that the second
kernel joins, row starts that decrease."""
import ctypes

import pytest
import torch

from paper_2604_00529_b200.binding import FORMATS, _Batch, _Cache, _Rows

from test_debug_build import P, report, u8
from test_debug_cache import D  # noqa: F401
from test_debug_products import clean, some

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


class Batch:
    """Exactly sized buffers of a cache and a batch; the binding's structs over them."""

    def __init__(self, lengths, starts, tokens, page, dim, block, heads, fmt, bits):
        need = [-(-n // page) for n in lengths]
        self.pages, width, batch = sum(need), max(need), len(lengths)
        n = self.pages * heads * page * dim
        self.bufs = some(n * bits // 8), some(n // block), some(n * bits // 8), some(n // block)
        table, at = torch.full((batch, width), -1, dtype=torch.int32), 0
        for b, m in enumerate(need):
            table[b, :m] = torch.arange(at, at + m)
            at += m
        self.arrays = table.cuda(), ints(lengths), ints(starts)
        self.cache = _Cache(*[P(t) for t in self.bufs], self.pages, page, heads, dim, FORMATS[fmt], block)
        self.batch = _Batch(*[P(t) for t in self.arrays], batch, width)
        self.tokens, self.heads, self.dim = tokens, heads, dim

    def attend(self, D, dtype, group, window):  # noqa: F811
        q_heads, size = self.heads * group, 4 if dtype == 0 else 2
        n = self.tokens * q_heads
        q, out, lse = some(n * self.dim * size), u8(n * self.dim * size), u8(n * 4)
        rows = _Rows(P(q), q_heads * self.dim, self.dim)
        need = D.mxq_cache_attention_workspace_bytes(ctypes.byref(self.cache), ctypes.byref(self.batch), q_heads, dtype, self.tokens)
        ws = u8(need)
        assert D.mxq_cache_attention(ctypes.byref(self.cache), ctypes.byref(self.batch), ctypes.byref(rows), q_heads, dtype, self.tokens, 0.1, 1, window,
                                     P(out), P(lse), P(ws), need, torch.cuda.current_stream().cuda_stream) == 0


@pytest.mark.parametrize("fmt,bits", [("e4m3", 8), ("int4", 4)])
@pytest.mark.parametrize("starts", [[0, 5, 2, 9], [9, 0, 9, 3], [-3, 4, 100, 2], [7, 7, 7, 7], [8, 6, 4, 2]])
def test_starts_that_decrease(D, starts, fmt, bits):  # noqa: F811
    for tokens, group in ((9, 1), (90, 2)):                  # few rows and many
        b = Batch([40, 3000, 70], [s * tokens // 9 for s in starts], tokens, 32, 64, 32, 2, fmt, bits)
        report(D)
        for dtype in (0, 1):
            for window in (0, 50):
                b.attend(D, dtype, group, window)
            kv = some(tokens * 2 * 64 * (4 if dtype == 0 else 2))
            r = _Rows(P(kv), 128, 64)
            stream = torch.cuda.current_stream().cuda_stream
            assert D.mxq_cache_write(ctypes.byref(b.cache), ctypes.byref(b.batch), ctypes.byref(r), ctypes.byref(r), dtype, tokens, stream) == 0
            assert D.mxq_cache_read(ctypes.byref(b.cache), ctypes.byref(b.batch), tokens, P(kv), P(kv), dtype, stream) == 0
        clean(D, 6)


@pytest.mark.parametrize("fmt,bits", [("e4m3", 8), ("e2m1", 4), ("int8", 8), ("int4", 4)])
@pytest.mark.parametrize("counts,lengths,page,dim,block,heads,group", [
    ([1], [9000], 64, 128, 32, 2, 4), ([1, 1, 1], [20000, 3, 700], 128, 64, 32, 1, 16), ([3, 2], [3000, 6000], 32, 256, 64, 1, 3),
    ([300], [5000], 64, 128, 64, 2, 2), ([130, 0, 200], [4000, 9, 210], 16, 64, 64, 3, 1)])
def test_windows_and_items_in_parts(D, counts, lengths, page, dim, block, heads, group, fmt, bits):  # noqa: F811
    b = Batch(lengths, [sum(counts[:i]) for i in range(len(counts) + 1)], sum(counts), page, dim, block, heads, fmt, bits)
    for dtype in (0, 1):
        for window in (0, 1, 100, 2500):
            report(D)
            b.attend(D, dtype, group, window)
            clean(D, 2)                                      # the items' kernel and the one that joins parts
