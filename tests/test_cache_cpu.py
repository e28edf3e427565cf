"""Refusals of the operators over a paged cache of codes: every call here is answered on the host, before any launch."""
import ctypes as C

import pytest
import torch

import paper_2604_00529_b200 as mxq
from paper_2604_00529_b200.binding import _Batch, _Cache, _Rows

OK, E_NULL, E_FORMAT, E_BLOCK, E_SIZE, E_ALIGN = 0, -1, -2, -3, -4, -5
A = 0x1000                                   # aligned, never dereferenced
F = mxq.FORMATS
BIG = 1 << 40


@pytest.fixture(scope="module")
def L():
    return mxq.load_library()


def cache(**kw):
    d = dict(k_codes=A, k_scales=A, v_codes=A, v_scales=A, pages=8, page=64, heads=2, head_dim=128, fmt=F["e2m1"], block=32)
    d.update(kw)
    return _Cache(*d.values())


def batch(**kw):
    d = dict(table=A, lengths=A, starts=A, batch=4, width=2)
    d.update(kw)
    return _Batch(*d.values())


def rows(**kw):
    d = dict(data=A, token_stride=256, head_stride=128)
    d.update(kw)
    return _Rows(*d.values())


def write(L, c=None, b=None, k=None, v=None, dtype=1, tokens=4):
    return L.mxq_cache_write(C.byref(c or cache()), C.byref(b or batch()), C.byref(k or rows()), C.byref(v or rows()), dtype, tokens, None)


def read(L, c=None, b=None, total=4, k=A, v=A, dtype=1):
    return L.mxq_cache_read(C.byref(c or cache()), C.byref(b or batch()), total, k, v, dtype, None)


def attend(L, c=None, b=None, q=None, q_heads=4, dtype=1, tokens=4, causal=1, window=0, out=A, lse=None, ws=A, ws_bytes=BIG):
    return L.mxq_cache_attention(C.byref(c or cache()), C.byref(b or batch()), C.byref(q or rows(token_stride=512)), q_heads, dtype, tokens, 0.1, causal,
                                 window, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [write, read, attend])
def test_descriptions(L, call):
    for fmt, i in F.items():
        if fmt not in ("e4m3", "e2m1", "int8", "int4"):
            assert call(L, cache(fmt=i)) == E_FORMAT
    assert call(L, cache(fmt=99)) == E_FORMAT and call(L, dtype=2) == E_FORMAT
    for block in (0, -32, 16, 48, 256):
        assert call(L, cache(block=block)) == E_BLOCK
    for dim in (0, 32, 96, 192, 512):
        assert call(L, cache(head_dim=dim)) == E_SIZE
    assert call(L, cache(head_dim=64, block=128)) == E_SIZE
    for page in (0, 8, 48, 512, -64):
        assert call(L, cache(page=page)) == E_SIZE
    assert call(L, cache(heads=0)) == E_SIZE and call(L, cache(heads=1025), **({"q_heads": 1025} if call is attend else {})) == E_SIZE
    assert call(L, cache(pages=1 << 31)) == E_SIZE
    for name in ("k_codes", "v_codes"):
        assert call(L, cache(**{name: None})) == E_NULL and call(L, cache(**{name: A + 16})) == E_ALIGN
    for name in ("k_scales", "v_scales"):
        assert call(L, cache(**{name: None})) == E_NULL and call(L, cache(**{name: A + 8})) == E_ALIGN
    assert call(L, None, batch(table=None)) == E_NULL and call(L, None, batch(table=A + 2)) == E_ALIGN
    assert call(L, None, batch(starts=A + 2)) == E_ALIGN
    assert call(L, None, batch(width=1 << 31)) == E_SIZE and call(L, None, batch(batch=1 << 31)) == E_SIZE
    if call is not read:
        assert call(L, None, batch(lengths=None)) == E_NULL and call(L, None, batch(lengths=A + 1)) == E_ALIGN
        assert call(L, None, batch(starts=None), tokens=5) == E_SIZE
    else:
        assert call(L, None, batch(starts=None)) == E_NULL


def test_null_structs(L):
    c, b, r = C.byref(cache()), C.byref(batch()), C.byref(rows())
    assert L.mxq_cache_write(None, b, r, r, 1, 4, None) == E_NULL and L.mxq_cache_write(c, None, r, r, 1, 4, None) == E_NULL
    assert L.mxq_cache_write(c, b, None, r, 1, 4, None) == E_NULL and L.mxq_cache_write(c, b, r, None, 1, 4, None) == E_NULL
    assert L.mxq_cache_read(None, b, 4, A, A, 1, None) == E_NULL and L.mxq_cache_read(c, None, 4, A, A, 1, None) == E_NULL
    assert L.mxq_cache_attention(None, b, r, 4, 1, 4, 0.1, 1, 0, A, None, A, BIG, None) == E_NULL
    assert L.mxq_cache_attention(c, b, None, 4, 1, 4, 0.1, 1, 0, A, None, A, BIG, None) == E_NULL
    assert L.mxq_cache_attention_workspace_bytes(None, b, 4, 1, 4) == 0


def test_rows_and_outputs(L):
    for bad, want in ((rows(data=None), E_NULL), (rows(data=A + 16), E_ALIGN), (rows(token_stride=8), E_ALIGN), (rows(head_stride=24), E_ALIGN)):
        assert write(L, k=bad) == want and write(L, v=bad) == want and attend(L, q=bad) == want
    assert read(L, k=None) == E_NULL and read(L, v=A + 16) == E_ALIGN
    assert attend(L, out=None) == E_NULL and attend(L, out=A + 16) == E_ALIGN and attend(L, lse=A + 2) == E_ALIGN
    assert attend(L, ws=None) == E_NULL and attend(L, ws=A + 8) == E_ALIGN and attend(L, ws_bytes=0) == E_SIZE
    assert attend(L, q_heads=3) == E_SIZE and attend(L, q_heads=0) == E_SIZE and attend(L, q_heads=(1 << 16) + 2) == E_SIZE
    assert attend(L, causal=0, window=5) == E_SIZE
    assert attend(L, tokens=1 << 25) == E_SIZE and attend(L, tokens=1 << 31) == E_SIZE      # more rows than MXQ_CACHE_ROWS_MAX


def test_nothing_to_do(L):
    none = cache(k_codes=None, k_scales=None, v_codes=None, v_scales=None)
    empty = batch(table=None, lengths=None, starts=None, batch=0, width=0)
    assert write(L, none, empty, rows(data=None), rows(data=None), tokens=0) == OK
    assert read(L, none, empty, 0, None, None) == OK
    assert attend(L, none, empty, rows(data=None), tokens=0, out=None, ws=None, ws_bytes=0) == OK


def test_workspace_covers_what_the_call_asks_for(L):
    for dim in (64, 128, 256):
        for tokens, n, width in ((1, 1, 1), (64, 64, 128), (300, 3, 40), (5, 1, 20000)):
            for dtype in (torch.bfloat16, torch.float32):
                need = mxq.cache_attention_workspace_bytes(tokens, 8, n, width, 64, 2, dim, dtype)
                assert need > 0
                b = batch(batch=n, width=width, starts=A)
                dt = 0 if dtype == torch.float32 else 1
                assert attend(L, cache(head_dim=dim), b, rows(token_stride=8 * dim, head_stride=dim), 8, dt, tokens, ws_bytes=need - 1) == E_SIZE
    assert mxq.cache_attention_workspace_bytes(1, 3, 1, 1, 64, 2, 128) == 0


def test_binding_refusals():
    with pytest.raises(mxq.MxqError):
        mxq.make_cache(4, 2, 128, "e3m2", device="cpu")
    with pytest.raises(mxq.MxqError):
        mxq.make_cache(4, 2, 128, "e2m1", block=16, device="cpu")
    with pytest.raises(mxq.MxqError):
        mxq.make_cache(4, 2, 96, "e2m1", device="cpu")
    bufs = mxq.make_cache(4, 2, 128, "int4", block=64, page=32, device="cpu")
    assert [tuple(t.shape) for t in bufs] == [(4, 2, 32, 64), (4, 2, 32, 2)] * 2 and not any(t.any() for t in bufs)
    k, table, lengths = torch.zeros(3, 2, 128), torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        mxq.cache_write(k, k, *bufs, table, lengths, "int4", block=64)                    # CPU tensors
    with pytest.raises(ValueError):
        mxq.cache_write(k, k, *bufs, table, lengths, "int4", block=32)                    # scales of another block size
    with pytest.raises(TypeError):
        mxq.cache_attention(k, bufs[0].float(), *bufs[1:], table, lengths, "int4", block=64)
    with pytest.raises(ValueError):
        mxq.cache_read(*bufs, table, torch.zeros(4, dtype=torch.int32), -1, "int4", block=64)
