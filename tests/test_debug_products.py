"""The operators that multiply by stored codes in the bounds-checked build: sizes where index arithmetic goes wrong first, with exactly
sized buffers; every plain access of the kernels lies in the buffers that the call was given."""
import ctypes
import os

import pytest
import torch

from paper_2604_00529_b200.binding import FORMATS, _MoeLayer

from test_debug_build import LIB, Info, P, report, u8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    if not os.path.exists(LIB):
        pytest.fail("libmxq_debug.so is not built: python -m paper_2604_00529_b200.build --debug")
    L = ctypes.CDLL(LIB)
    vp, sz, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    L.mxq_matmul.argtypes = [vp, vp, vp, vp, sz, sz, sz, i, i, vp, i, vp]
    L.mxq_matrix_codes_bytes.argtypes = L.mxq_matrix_scales_bytes.argtypes = [sz, sz, i]
    L.mxq_matrix_codes_bytes.restype = L.mxq_matrix_scales_bytes.restype = sz
    L.mxq_quantize_matrix.argtypes = [vp, i, sz, sz, i, i, vp, vp, vp, vp, vp]
    L.mxq_moe_workspace_bytes.argtypes = [sz, i, sz, i]
    L.mxq_moe_workspace_bytes.restype = sz
    L.mxq_moe.argtypes = [ctypes.POINTER(_MoeLayer), vp, i, vp, sz, i, i, vp, vp, sz, vp]
    L.mxq_debug_report.argtypes = [ctypes.POINTER(Info), i]
    return L


def clean(D, launches):
    info = report(D)
    assert info.enabled == 1 and info.checked_launches >= launches
    assert info.violations == 0, "%d accesses outside, the first at %#x" % (info.violations, info.first_address)


def some(nbytes, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 120, (nbytes,), generator=g, device="cuda", dtype=torch.uint8)


@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 130), (33, 32), (128, 128), (129, 257), (200, 72)])
def test_quantize_matrix_stays_inside(D, rows, cols, block, dtype, size):
    stream = torch.cuda.current_stream().cuda_stream
    report(D)
    src = torch.zeros(rows * cols * size, dtype=torch.uint8, device="cuda")
    cb, sb = D.mxq_matrix_codes_bytes, D.mxq_matrix_scales_bytes
    outs = [u8(cb(rows, cols, block)), u8(sb(rows, cols, block)), u8(cb(cols, rows, block)), u8(sb(cols, rows, block))]
    assert D.mxq_quantize_matrix(P(src), dtype, rows, cols, 3, block, *[P(t) for t in outs], stream) == 0
    clean(D, 1)


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(1, 1, 128), (1, 17, 384), (8, 16, 128), (9, 33, 1152), (17, 40, 128), (70, 130, 256), (300, 260, 128)])
def test_matmul_stays_inside(D, m, n, k, block):
    stream = torch.cuda.current_stream().cuda_stream
    for dtype, size in ((0, 4), (1, 2)):
        report(D)
        a, b, sa, sb = some(m * k), some(n * k), some(m * k // block), some(n * k // block)
        out = u8(m * n * size)
        assert D.mxq_matmul(P(a), P(sa), P(b), P(sb), m, n, k, 3, block, P(out), dtype, stream) == 0
        clean(D, 1)


@pytest.mark.parametrize("fmt,bits", [("e4m3", 8), ("e2m1", 4), ("int8", 8), ("int4", 4)])
@pytest.mark.parametrize("tokens,experts,top_k,hidden,inner,block", [(1, 1, 1, 32, 32, 32), (3, 5, 2, 96, 160, 32), (64, 3, 3, 128, 64, 64),
                                                                   (17, 40, 6, 128, 128, 128), (2, 512, 16, 64, 96, 32)])
def test_moe_stays_inside(D, tokens, experts, top_k, hidden, inner, block, fmt, bits):
    stream = torch.cuda.current_stream().cuda_stream
    for dtype, size in ((0, 4), (1, 2)):
        report(D)
        w = experts * hidden * inner
        up, us, dn, ds = some(2 * w * bits // 8), some(2 * w // block), some(w * bits // 8), some(w // block)
        x, out = torch.zeros(tokens * hidden * size, dtype=torch.uint8, device="cuda"), u8(tokens * hidden * size)
        lg = torch.randn(tokens, experts, device="cuda")
        need = D.mxq_moe_workspace_bytes(tokens, top_k, inner, dtype)
        ws = u8(need)
        layer = _MoeLayer(P(up), P(us), P(dn), P(ds), hidden, inner, experts, FORMATS[fmt], block)
        assert D.mxq_moe(ctypes.byref(layer), P(x), dtype, P(lg), tokens, top_k, 1, P(out), P(ws), need, stream) == 0
        clean(D, 2)
