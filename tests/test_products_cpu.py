"""Refusals of the operators that multiply by stored codes: every call here is answered on the host, before any launch."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq
from paper_2604_00529_b200.binding import _MoeLayer

import product_util as pu
from oracle import mxq_oracle as orc

OK, E_NULL, E_FORMAT, E_BLOCK, E_SIZE, E_ALIGN = 0, -1, -2, -3, -4, -5
A = 0x1000                                   # aligned, never dereferenced
F = mxq.FORMATS


@pytest.fixture(scope="module")
def L():
    return mxq.load_library()


def test_matmul_refusals(L):
    mm = L.mxq_matmul                        # (a, as, b, bs, m, n, k, fmt, block, dst, dtype, stream)
    e4 = F["e4m3"]
    for fmt in F.values():
        if fmt != e4:
            assert mm(A, A, A, A, 4, 4, 128, fmt, 128, A, 1, None) == E_FORMAT
    assert mm(A, A, A, A, 4, 4, 128, 99, 128, A, 1, None) == E_FORMAT
    assert mm(A, A, A, A, 4, 4, 128, e4, 128, A, 2, None) == E_FORMAT
    for block in (0, -32, 16, 48, 256):
        assert mm(A, A, A, A, 4, 4, 768, e4, block, A, 1, None) == E_BLOCK
    assert mm(A, A, A, A, 4, 4, 96, e4, 64, A, 1, None) == E_SIZE
    assert mm(A, A, A, A, 1 << 31, 4, 128, e4, 128, A, 1, None) == E_SIZE
    assert mm(A, A, A, A, 4, 1 << 31, 128, e4, 128, A, 1, None) == E_SIZE
    assert mm(A, A, A, A, 4, 4, 1 << 31, e4, 128, A, 1, None) == E_SIZE
    assert mm(None, None, None, None, 0, 4, 128, e4, 128, None, 1, None) == OK
    assert mm(None, None, None, None, 4, 0, 128, e4, 128, None, 1, None) == OK
    for at in range(4):
        args = [A] * 4
        args[at] = None
        assert mm(*args, 4, 4, 128, e4, 128, A, 1, None) == E_NULL
        args[at] = A + 8
        assert mm(*args, 4, 4, 128, e4, 128, A, 1, None) == E_ALIGN
    assert mm(A, A, A, A, 4, 4, 128, e4, 128, None, 1, None) == E_NULL
    assert mm(None, None, None, None, 4, 4, 0, e4, 128, None, 1, None) == E_NULL
    assert mm(A, A, A, A, 4, 4, 128, e4, 128, A + 16, 1, None) == E_ALIGN


def test_quantize_matrix_refusals(L):
    q = L.mxq_quantize_matrix                # (src, dtype, rows, cols, fmt, block, codes, scales, codes_t, scales_t, stream)
    e4 = F["e4m3"]
    assert q(A, 1, 4, 4, F["int8"], 32, A, A, A, A, None) == E_FORMAT
    assert q(A, 3, 4, 4, e4, 32, A, A, A, A, None) == E_FORMAT
    assert q(A, 1, 4, 4, e4, 16, A, A, A, A, None) == E_BLOCK
    assert q(A, 1, 4, 4, e4, 32, None, None, None, None, None) == E_NULL
    assert q(None, 1, 4, 4, e4, 32, A, A, A, A, None) == E_NULL
    assert q(A, 1, 4, 4, e4, 32, A, None, A, A, None) == E_NULL
    assert q(A, 1, 4, 4, e4, 32, A, A, None, A, None) == E_NULL
    assert q(A + 16, 1, 4, 4, e4, 32, A, A, A, A, None) == E_ALIGN
    assert q(A, 1, 4, 4, e4, 32, A + 16, A, A, A, None) == E_ALIGN
    assert q(A, 1, 4, 4, e4, 32, A, A, A, A + 8, None) == E_ALIGN
    assert q(A, 1, 1 << 40, 1 << 40, e4, 32, A, A, A, A, None) == E_SIZE
    assert q(None, 1, 0, 4, e4, 32, None, None, None, None, None) == OK
    assert q(None, 1, 4, 0, e4, 32, None, None, None, None, None) == OK
    assert L.mxq_matrix_codes_bytes(5, 33, 32) == 5 * 64 and L.mxq_matrix_scales_bytes(5, 33, 32) == 10
    assert L.mxq_matrix_codes_bytes(5, 128, 128) == 640 and L.mxq_matrix_codes_bytes(5, 33, 0) == 0


def _layer(**kw):
    d = dict(up_codes=A, up_scales=A, down_codes=A, down_scales=A, hidden=128, inner=64, experts=4, fmt=F["e4m3"], block=32)
    d.update(kw)
    return _MoeLayer(**d)


def test_moe_refusals(L):
    big = 1 << 30

    def call(layer=None, x=A, dtype=1, logits=A, tokens=2, top_k=2, out=A, ws=A, ws_bytes=big):
        return L.mxq_moe(C.byref(layer if layer is not None else _layer()), x, dtype, logits, tokens, top_k, 1, out, ws, ws_bytes, None)

    assert L.mxq_moe(None, A, 1, A, 2, 2, 1, A, A, big, None) == E_NULL
    for fmt in ("int7", "int6", "int5", "int3", "int2", "e3m3", "e3m2", "e2m3", "e2m2"):
        assert call(_layer(fmt=F[fmt])) == E_FORMAT
    assert call(dtype=2) == E_FORMAT
    assert call(_layer(block=16)) == E_BLOCK and call(_layer(block=0)) == E_BLOCK
    assert call(_layer(hidden=144)) == E_SIZE and call(_layer(inner=80)) == E_SIZE
    assert call(_layer(hidden=0)) == E_SIZE and call(_layer(inner=0)) == E_SIZE
    assert call(_layer(hidden=(1 << 20) + 32)) == E_SIZE
    assert call(_layer(experts=0)) == E_SIZE and call(_layer(experts=513)) == E_SIZE
    assert call(tokens=65) == E_SIZE
    assert call(top_k=0) == E_SIZE and call(top_k=5) == E_SIZE and call(_layer(experts=32), top_k=17) == E_SIZE
    assert call(ws_bytes=mxq.moe_workspace_bytes(2, 2, 64) - 1) == E_SIZE
    for name in ("x", "logits", "out", "ws"):
        assert call(**{name: None}) == E_NULL
        assert call(**{name: A + 2}) == E_ALIGN
    for name in ("up_codes", "up_scales", "down_codes", "down_scales"):
        assert call(_layer(**{name: None})) == E_NULL
        assert call(_layer(**{name: A + 8})) == E_ALIGN
    assert call(tokens=0, x=None, logits=None, out=None, ws=None) == OK


def test_moe_workspace_bytes():
    assert mxq.moe_workspace_bytes(0, 2, 64) == 0
    assert mxq.moe_workspace_bytes(3, 2, 96) >= 3 * 2 * 96 * 4
    assert mxq.moe_workspace_bytes(3, 2, 96, torch.float32) >= 3 * 2 * 96 * 6
    assert mxq.moe_workspace_bytes(65, 2, 64) == 0 and mxq.moe_workspace_bytes(2, 17, 64) == 0


def test_binding_refusals():
    c, s = torch.zeros(4 * 128, dtype=torch.uint8), torch.zeros(4, dtype=torch.uint8)
    with pytest.raises(ValueError):
        mxq.matmul(c, s, c, s, 4, 4, 128, block=128)                    # CPU tensors
    with pytest.raises(ValueError):
        mxq.matmul(c, s, c, s, 8, 4, 128, block=128)                    # too few codes
    with pytest.raises(ValueError):
        mxq.matmul(c, s, c, s, -1, 4, 128, block=128)
    with pytest.raises(TypeError):
        mxq.matmul(c.float(), s, c, s, 4, 4, 128, block=128)
    with pytest.raises(ValueError):
        mxq.quantize_matrix(torch.zeros(4, 4))
    with pytest.raises(ValueError):
        mxq.quantize_matrix(torch.zeros(4))
    with pytest.raises(ValueError):
        mxq.linear_ste(torch.zeros(4, 32), torch.zeros(8, 32))
    with pytest.raises(ValueError):
        mxq.linear_ste(torch.zeros(4, 32), torch.zeros(8, 33))
    with pytest.raises(TypeError):
        mxq.linear_ste(torch.zeros(4, 32, dtype=torch.float16), torch.zeros(8, 32))
    with pytest.raises(mxq.MxqError):
        mxq.linear_ste(torch.zeros(4, 32), torch.zeros(8, 32), block=16)
    x, lg = torch.zeros(2, 64), torch.zeros(2, 4)
    up, us = torch.zeros(4 * 2 * 32 * 64, dtype=torch.uint8), torch.zeros(4 * 2 * 32 * 2, dtype=torch.uint8)
    dn, ds = torch.zeros(4 * 32 * 64, dtype=torch.uint8), torch.zeros(4 * 64, dtype=torch.uint8)
    with pytest.raises(ValueError):
        mxq.moe(x, lg, up, us, dn, ds, 32, 2, "e4m3")
    with pytest.raises(TypeError):
        mxq.moe(x, lg.bfloat16(), up, us, dn, ds, 32, 2, "e4m3")
    with pytest.raises(ValueError):
        mxq.moe(x, lg[:1], up, us, dn, ds, 32, 2, "e4m3")
    with pytest.raises(ValueError):
        mxq.moe(x, lg, up[:-1], us, dn, ds, 32, 2, "e4m3")


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1", "int8", "int4"])
def test_the_plain_values_are_the_oracles(fmt):
    """The 64-bit values that the GPU tests compare with, against the oracle's reconstruction."""
    rng = np.random.default_rng(3)
    packed, scales, want = pu.quantized(rng, 4, 128, fmt, 32)
    codes = orc.unpack(packed, 4 * 128, orc.bits(fmt))
    got = orc.dequantize(codes, scales.reshape(-1), fmt).reshape(4, 128)
    assert np.array_equal(got.astype(np.float64), want)


def test_the_plain_choice():
    lg = np.array([[1.0, 3.0, 3.0, -np.inf], [-np.inf] * 4, [0.0, np.nan, 1.0, 2.0], [-np.inf, 0.0, -np.inf, -np.inf]])
    got = pu.choice64(lg, 2, True)
    assert [e for e, _ in got[0]] == [1, 2] and got[1] == [] and got[2] is None and got[3] == [(1, 1.0)]
    assert abs(sum(w for _, w in pu.choice64(lg, 2, False)[0]) - 2 / (2 + np.exp(-2.0))) < 1e-12
