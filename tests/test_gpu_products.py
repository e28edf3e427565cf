"""The operators that multiply by stored codes against their definitions in 64 bits: matmul, quantize_matrix, linear_ste, moe.
Where the tolerances come from: product_util."""
import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq
import paper_2604_00529_b200.binding  # noqa: F401
from oracle import mxq_oracle as orc

import product_util as pu
from gpu_util import Guarded, to_dev, to_host

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def rng_of(*key):
    return np.random.default_rng(list(key))


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- matmul ---------------------------------------------------------------------------------------------------

MATMUL = [(1, 1, 128), (1, 17, 384), (1, 4096, 256), (7, 16, 640), (8, 33, 128), (9, 100, 1152), (16, 31, 2048), (17, 257, 384),
          (33, 130, 1152), (64, 64, 128), (65, 129, 512), (127, 40, 256), (130, 300, 640), (200, 96, 4096), (257, 513, 384), (600, 700, 1024)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", MATMUL)
def test_matmul(m, n, k, block, dtype):
    rng = rng_of(m, n, k, block)
    ac, as_, a = pu.quantized(rng, m, k, "e4m3", block)
    bc, bs, b = pu.quantized(rng, n, k, "e4m3", block, 0.02)
    out = Guarded(m * n * dtype.itemsize, dtype)
    got = mxq.matmul(dev(ac), dev(as_), dev(bc), dev(bs), m, n, k, block=block, out=out.view)
    out.check()
    pu.check(got.view(m, n), a @ b.T, pu.sum_bound(k, np.abs(a) @ np.abs(b).T))


@pytest.mark.parametrize("m,n,k,block", [(5, 40, 96, 32), (20, 40, 1120, 32), (300, 260, 1120, 32), (300, 260, 192, 64)])
def test_matmul_k_beyond_whole_tiles(m, n, k, block):
    rng = rng_of(m, n, k, block)
    ac, as_, a = pu.quantized(rng, m, k, "e4m3", block)
    bc, bs, b = pu.quantized(rng, n, k, "e4m3", block)
    # what lies behind the operands must not matter
    pad = torch.full((4096,), 0x7E, dtype=torch.uint8, device="cuda")
    full = [torch.cat((dev(t.reshape(-1)), pad)) for t in (ac, as_, bc, bs)]
    got = mxq.matmul(*full, m, n, k, block=block, dtype=FP)
    pu.check(got, a @ b.T, pu.sum_bound(k, np.abs(a) @ np.abs(b).T))


@pytest.mark.parametrize("m", [1, 12, 150, 300])
@pytest.mark.parametrize("block", [32, 128])
def test_matmul_scales_at_the_ends_of_their_range(m, block):
    """Scale bytes from 0 to 254 whose products stay in FP32's range, and poisoned blocks."""
    rng, n, k = rng_of(m, block), 140, 256
    ac, _, _ = pu.quantized(rng, m, k, "e4m3", block)
    bc, _, _ = pu.quantized(rng, n, k, "e4m3", block)
    sa = rng.integers(0, 255, (m, 1)) + np.zeros((m, k // block), int)
    sa[:, 0] = np.clip(sa[:, 0] + rng.integers(-3, 4, m), 0, 254)
    sb = np.clip(236 + rng.integers(0, 4, (n, k // block)), 0, 254)
    sa = np.clip(sa, 0, 100)                                # sums of 256 products below 2^18 each stay finite
    sa[m // 2, 0] = 255
    sb[n // 3, -1] = 255
    a = pu.values64(ac.astype(np.int64).reshape(m, k), sa, "e4m3", block)
    b = pu.values64(bc.astype(np.int64).reshape(n, k), sb, "e4m3", block)
    got = mxq.matmul(dev(ac), dev(sa.astype(np.uint8)), dev(bc), dev(sb.astype(np.uint8)), m, n, k, block=block, dtype=FP)
    want = a @ b.T
    pu.check(got, want, np.nan_to_num(pu.sum_bound(k, np.abs(a) @ np.abs(b).T)))


@pytest.mark.parametrize("m,n,k,block,dtype", [(520, 4100, 640, 32, BF), (520, 4111, 1280, 128, FP), (2100, 4400, 512, 64, BF), (2100, 4401, 384, 128, BF),
                                               (2100, 4401, 192, 64, FP), (4100, 2500, 1152, 32, FP), (8200, 300, 256, 128, BF)])
def test_matmul_many_tiles(m, n, k, block, dtype):
    """Sizes at which a CTA works on several tiles in turn, whole and cut off."""
    rng = rng_of(m, n, k, block)
    ac, as_, a = pu.quantized(rng, m, k, "e4m3", block)
    bc, bs, b = pu.quantized(rng, n, k, "e4m3", block, 0.02)
    out = Guarded(m * n * dtype.itemsize, dtype)
    got = mxq.matmul(dev(ac), dev(as_), dev(bc), dev(bs), m, n, k, block=block, out=out.view)
    out.check()
    pu.check(got.view(m, n), a @ b.T, pu.sum_bound(k, np.abs(a) @ np.abs(b).T))
    again = mxq.matmul(dev(ac), dev(as_), dev(bc), dev(bs), m, n, k, block=block, dtype=dtype)
    assert torch.equal(got.view(m, n), again)


@pytest.mark.parametrize("m", [1, 20, 300])
def test_matmul_zero_blocks_against_the_largest_scales(m):
    """A block of zeros (scale byte 0) met by scales of 2^127, and the other way round: zeros, of either sign, not NaN."""
    n, k = 200, 128
    zero, low = torch.zeros(m * k, dtype=torch.uint8, device="cuda"), torch.zeros(m, dtype=torch.uint8, device="cuda")
    big, high = torch.full((n * k,), 0x7E, dtype=torch.uint8, device="cuda"), torch.full((n,), 254, dtype=torch.uint8, device="cuda")
    got = mxq.matmul(zero, low, big, high, m, n, k, block=128, dtype=FP)
    assert torch.equal(got, torch.zeros_like(got))
    got = mxq.matmul(big, high, zero, low, n, m, k, block=128)
    assert torch.equal(got, torch.zeros_like(got))


def test_no_wait_ran_out():
    a, s = torch.full((300 * 256,), 0x38, dtype=torch.uint8, device="cuda"), torch.full((600,), 127, dtype=torch.uint8, device="cuda")
    got = mxq.matmul(a, s, a, s, 300, 300, 256, block=128, dtype=FP)
    assert bool((got == 256).all())
    assert mxq.load_library().mxq_wait_status(1) == 0


def test_matmul_empty():
    c, s = torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")
    assert mxq.matmul(c, s, c, s, 0, 0, 128, block=128).shape == (0, 0)
    got = mxq.matmul(c, s, c, s, 3, 5, 0, block=128, out=torch.full((3, 5), 7.0, device="cuda"))
    assert torch.equal(got, torch.zeros(3, 5, device="cuda"))


def test_matmul_rows_do_not_depend_on_their_neighbours():
    """Each row of D is the same whatever rows stand beside it in calls of the same kind: padded batches."""
    rng, n, k = rng_of(5, 5), 96, 512
    ac, as_, _ = pu.quantized(rng, 300, k, "e4m3", 128)
    bc, bs, _ = pu.quantized(rng, n, k, "e4m3", 128)
    b = dev(bc), dev(bs)
    full = mxq.matmul(dev(ac), dev(as_), *b, 300, n, k, block=128)
    ac2, as2 = ac.copy().reshape(300, k), as_.copy()
    ac2[150:], as2[150:] = 0x7E, 200
    part = mxq.matmul(dev(ac2), dev(as2), *b, 300, n, k, block=128)
    assert torch.equal(full[:150], part[:150])


def test_matmul_offsets_beyond_32_bits():
    m, n, k = 3, (1 << 20) + 40, 4224                       # n * k passes 2^32
    rng = rng_of(1, 2)
    ac, as_, a = pu.quantized(rng, m, k, "e4m3", 128)
    tail = 300
    bc, bs, b = pu.quantized(rng, tail, k, "e4m3", 128)
    codes = torch.zeros(n * k, dtype=torch.uint8, device="cuda")
    scales = torch.full((n * k // 128,), 127, dtype=torch.uint8, device="cuda")
    codes[-tail * k:] = dev(bc.reshape(-1))
    scales[-tail * k // 128:] = dev(bs.reshape(-1))
    for rows in (1, 3):
        got = mxq.matmul(dev(ac), dev(as_), codes, scales, rows, n, k, block=128)
        assert not got[:, :-tail].any()
        pu.check(got[:, -tail:], a[:rows] @ b.T, pu.sum_bound(k, np.abs(a[:rows]) @ np.abs(b).T))
    # the long operand as the first one: 70 rows of the other
    ac, as_, a = pu.quantized(rng, 70, k, "e4m3", 128)
    got = mxq.matmul(codes, scales, dev(ac), dev(as_), n, 70, k, block=128)
    assert not got[:-tail].any()
    pu.check(got[-tail:], b @ a.T, pu.sum_bound(k, np.abs(b) @ np.abs(a).T))


@pytest.mark.parametrize("m", [3, 40, 300])
def test_matmul_on_another_stream_and_captured(m):
    rng, n, k = rng_of(m, 9), 272, 1024
    ac, as_, _ = pu.quantized(rng, m, k, "e4m3", 64)
    bc, bs, _ = pu.quantized(rng, n, k, "e4m3", 64)
    ops = [dev(t) for t in (ac, as_, bc, bs)]
    want = mxq.matmul(*ops, m, n, k, block=64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = mxq.matmul(*ops, m, n, k, block=64, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    assert torch.equal(mxq.matmul(*ops, m, n, k, block=64, stream=torch.cuda.current_stream()), want)
    assert torch.equal(mxq.matmul(*ops, m, n, k, block=64, stream=torch.cuda.current_stream().cuda_stream), want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    out = torch.empty(m, n, dtype=BF, device="cuda")
    with torch.cuda.graph(graph):
        mxq.matmul(*ops, m, n, k, block=64, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


# ---- quantize_matrix ------------------------------------------------------------------------------------------


def oracle_rows(x: np.ndarray, block: int):
    """Oracle bytes of x [rows, cols] (float32, or BF16 patterns) along its rows, padded with zeros to whole blocks."""
    p = np.pad(x, ((0, 0), (0, -x.shape[1] % block)))
    codes, scales = orc.quantize(np.ascontiguousarray(p).reshape(-1), "e4m3", block)
    return np.asarray(codes).astype(np.uint8), np.asarray(scales)


def awkward(rng, rows, cols, dtype):
    x = (rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-20, 20, (rows, cols)))).astype(np.float32)
    x[rng.random((rows, cols)) < 0.02] = 0.0
    x[rng.random((rows, cols)) < 0.02] = -0.0
    x[rng.random((rows, cols)) < 0.01] = 1e-41                # an FP32 subnormal
    if rows * cols > 500:
        x[rows // 2, cols // 3] = np.inf
        x[rows // 3, cols // 2] = np.nan
        x[rows - 1, cols - 1] = -3.3e38
    if dtype == BF:
        return (x.view(np.uint32) >> 16).astype(np.uint16)    # cut to BF16 patterns
    return x


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 200), (31, 33), (64, 64), (128, 128), (129, 257), (300, 1000), (1000, 72)])
def test_quantize_matrix(rows, cols, block, dtype):
    x = awkward(rng_of(rows, cols, block), rows, cols, dtype)
    src = to_dev(x)
    wr, wc = oracle_rows(x, block), oracle_rows(np.ascontiguousarray(x.T), block)
    got = mxq.quantize_matrix(src, block=block)
    for g, w, what in zip(got, wr + wc, ("codes", "scales", "codes_t", "scales_t")):
        assert np.array_equal(to_host(g), w), what
    only = mxq.quantize_matrix(src, block=block, cols=False)
    assert only[2] is None and only[3] is None and torch.equal(only[0], got[0]) and torch.equal(only[1], got[1])
    only = mxq.quantize_matrix(src, block=block, rows=False)
    assert only[0] is None and only[1] is None and torch.equal(only[2], got[2]) and torch.equal(only[3], got[3])


def test_quantize_matrix_is_quantize_where_both_go():
    x = torch.randn(96, 256, device="cuda", dtype=BF)
    c, s, ct, st = mxq.quantize_matrix(x, block=32)
    wc, ws = mxq.quantize(x, "e4m3", 32)
    assert torch.equal(c, wc) and torch.equal(s, ws)
    wc, ws = mxq.quantize(x.t().contiguous(), "e4m3", 32)
    assert torch.equal(ct, wc) and torch.equal(st, ws)


def test_quantize_matrix_writes_its_buffers_only():
    L = mxq.load_library()
    rows, cols, block = 131, 77, 64
    x = torch.randn(rows, cols, device="cuda")
    outs = [Guarded(f(*d, block)) for d in ((rows, cols), (cols, rows)) for f in (L.mxq_matrix_codes_bytes, L.mxq_matrix_scales_bytes)]
    rc = L.mxq_quantize_matrix(x.data_ptr(), 0, rows, cols, 3, block, *[o.view.data_ptr() for o in outs], torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    want = mxq.quantize_matrix(x, block=block)
    for o, w in zip(outs, want):
        o.check()
        assert torch.equal(o.view, w)


# ---- linear_ste -----------------------------------------------------------------------------------------------


def linear64(x, w, dy, block):
    q = lambda v: pu.e4m3_64(np.ascontiguousarray(v), block)  # noqa: E731
    pairs = ((q(x), q(w)), (q(dy), q(w.T)), (q(dy.T), q(x.T)))
    return [(a @ b.T, pu.sum_bound(a.shape[1], np.abs(a) @ np.abs(b).T)) for a, b in pairs]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m,n,k,block", [(1, 1, 1, 32), (5, 70, 33, 32), (40, 64, 128, 64), (130, 96, 200, 128), (257, 300, 129, 32)])
def test_linear_ste(m, n, k, block, dtype):
    g = torch.Generator(device="cuda").manual_seed(m * n + k)
    x = torch.randn(m, k, generator=g, device="cuda").to(dtype).requires_grad_()
    w = (torch.randn(n, k, generator=g, device="cuda") * 0.1).to(dtype).requires_grad_()
    dy = (torch.randn(m, n, generator=g, device="cuda") * 1e-3).to(dtype)
    y = mxq.linear_ste(x, w, block)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    for got, (want, bound) in zip((y, dx, dw), linear64(pu.to64(x), pu.to64(w), pu.to64(dy), block)):
        assert got.dtype == dtype
        pu.check(got, want, bound)


def test_linear_ste_shapes_views_and_frozen_leaves():
    x = torch.randn(2, 3, 40, device="cuda", dtype=BF, requires_grad=True)
    w = torch.randn(40, 24, device="cuda", dtype=BF, requires_grad=True)
    y = mxq.linear_ste(x, w.t(), 32)                       # a transposed view of the weight
    assert y.shape == (2, 3, 24)
    y.backward(torch.ones_like(y))
    x2, w2 = x.detach().reshape(6, 40).requires_grad_(), w.detach().t().contiguous().requires_grad_()
    y2 = mxq.linear_ste(x2, w2, 32)
    y2.backward(torch.ones_like(y2))
    assert torch.equal(y.reshape(6, 24), y2) and torch.equal(x.grad.reshape(6, 40), x2.grad) and torch.equal(w.grad, w2.grad.t())
    x3 = x2.detach()                                        # no gradient for x, then none for w
    (gw,) = torch.autograd.grad(mxq.linear_ste(x3, w2, 32), w2, torch.ones_like(y2))
    assert torch.equal(gw, w2.grad)
    (gx,) = torch.autograd.grad(mxq.linear_ste(x2, w2.detach(), 32), x2, torch.ones_like(y2))
    assert torch.equal(gx, x2.grad)
    assert not mxq.linear_ste(x3, w2.detach(), 32).requires_grad


def test_linear_ste_parameters_shared_and_broadcast():
    """A parameter used twice, and one row broadcast over the batch: the gradients add up."""
    w = torch.nn.Parameter(torch.randn(48, 64, device="cuda") * 0.1)
    x = torch.randn(6, 64, device="cuda", requires_grad=True)
    dy = torch.randn(6, 48, device="cuda")
    (mxq.linear_ste(x, w) * dy).sum().backward()
    one_w, one_x = w.grad.clone(), x.grad.clone()
    w.grad = x.grad = None
    ((mxq.linear_ste(x, w) + mxq.linear_ste(x, w)) * dy).sum().backward()
    assert torch.equal(w.grad, 2 * one_w) and torch.equal(x.grad, 2 * one_x)
    row = torch.randn(1, 64, device="cuda", requires_grad=True)
    y = mxq.linear_ste(row.expand(6, 64), w)
    (g,) = torch.autograd.grad(y, row, dy)
    full = row.detach().repeat(6, 1).requires_grad_()
    (want,) = torch.autograd.grad(mxq.linear_ste(full, w), full, dy)
    assert torch.equal(g, want.sum(0, keepdim=True))


def test_linear_ste_gradients_against_differences():
    """On values that the format holds exactly the layer is bilinear, so whole steps give the gradient exactly."""
    rng = rng_of(8, 8)
    m, n, k = 6, 40, 32
    x = rng.integers(-3, 4, (m, k)).astype(np.float32)
    w = rng.integers(-3, 4, (n, k)).astype(np.float32)
    x[:, 0], w[:, 0], x[0], w[0] = 4, 4, 4, 4              # every block's largest value stays where it is
    dy = rng.integers(-3, 4, (m, n)).astype(np.float32)
    f = lambda x, w: float((pu.to64(mxq.linear_ste(dev(x), dev(w), 32)) * dy).sum())  # noqa: E731
    tx, tw = dev(x).requires_grad_(), dev(w).requires_grad_()
    dx, dw = torch.autograd.grad(mxq.linear_ste(tx, tw, 32), (tx, tw), dev(dy))
    for i, j in ((1, 1), (3, 7), (5, 31)):
        for at, grad in ((x, dx), (w, dw)):
            hi, lo = at.copy(), at.copy()
            hi[i, j] += 1
            lo[i, j] -= 1
            d = (f(hi, w) - f(lo, w)) / 2 if at is x else (f(x, hi) - f(x, lo)) / 2
            assert d == float(grad[i, j])


@pytest.mark.parametrize("native", [True, False])
def test_linear_ste_has_no_second_derivative(native, monkeypatch):
    if not native:
        monkeypatch.setattr(mxq.binding._host, "linear_ste", lambda *a: None)
    x = torch.randn(4, 32, device="cuda", requires_grad=True)
    w = torch.randn(8, 32, device="cuda", requires_grad=True)
    (g,) = torch.autograd.grad(mxq.linear_ste(x, w).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_native_and_general_path_agree(monkeypatch):
    """The binding's native code and the Python code behind it: the same bits."""
    rng = rng_of(81, 3)
    ac, as_, _ = pu.quantized(rng, 40, 256, "e4m3", 64)
    ops = [dev(t) for t in (ac, as_, ac, as_)]
    x = torch.randn(5, 7, 96, device="cuda", dtype=BF, requires_grad=True)
    w = torch.randn(50, 96, device="cuda", requires_grad=True)
    xm, lg, up, down = moe_case(rng, 4, 6, 64, 96, "int4", 32, BF)

    def everything():
        y = mxq.linear_ste(x, w)
        moe = mxq.moe(xm, dev(lg), up[0], up[1], down[0], down[1], 96, 2, "int4")
        return [mxq.matmul(*ops, 40, 40, 256, block=64, dtype=FP), *mxq.quantize_matrix(x.detach().view(35, 96)), moe, y.detach(),
                *torch.autograd.grad(y, (x, w), torch.ones_like(y))]

    native = everything()
    assert all(t.device.type == "cuda" for t in native)
    host = mxq.binding._host
    assert host.matmul(*ops, 40, 40, 256, "e4m3", 64, FP, None, None) is not None
    for name in ("matmul", "quantize_matrix", "moe", "linear_ste"):
        monkeypatch.setattr(host, name, lambda *a: None)
    for a, b in zip(native, everything()):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b)


def test_linear_ste_empty_batch():
    x = torch.empty(0, 64, device="cuda", requires_grad=True)
    w = torch.randn(48, 64, device="cuda", requires_grad=True)
    y = mxq.linear_ste(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), torch.empty(0, 48, device="cuda"))
    assert y.shape == (0, 48) and dx.shape == (0, 64) and torch.equal(dw, torch.zeros_like(w))


def test_linear_ste_step_captured_beside_an_eager_graph():
    """A step captured on the stream on which an eager graph of the same leaves was made and still lives, then replayed."""
    x = torch.randn(64, 96, device="cuda", dtype=BF, requires_grad=True)
    w = torch.randn(80, 96, device="cuda", dtype=BF, requires_grad=True)
    dy = torch.randn(64, 80, device="cuda", dtype=BF)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        alive = mxq.linear_ste(x, w)
        want = torch.autograd.grad(mxq.linear_ste(x, w), (x, w), dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = torch.autograd.grad(mxq.linear_ste(x, w), (x, w), dy)
    for _ in range(2):
        got[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with torch.cuda.stream(s):
        again = torch.autograd.grad(alive, (x, w), dy)
    torch.cuda.synchronize()
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


# ---- moe ------------------------------------------------------------------------------------------------------


def experts_of(rng, e, rows, k, fmt, block):
    packed, scales, values = pu.quantized(rng, e * rows, k, fmt, block, 0.1)
    return dev(packed), dev(scales), values.reshape(e, rows, k)


def moe_case(rng, t, e, hidden, inner, fmt, block, dtype):
    x = torch.from_numpy(rng.standard_normal((t, hidden)).astype(np.float32)).cuda().to(dtype)
    lg = (rng.standard_normal((t, e)) * 2).astype(np.float32)
    return x, lg, experts_of(rng, e, 2 * inner, hidden, fmt, block), experts_of(rng, e, hidden, inner, fmt, block)


def run_moe(x, lg, up, down, inner, top_k, fmt, block, renormalize=True):
    out = Guarded(x.numel() * x.element_size(), x.dtype)
    got = mxq.moe(x, dev(lg), up[0], up[1], down[0], down[1], inner, top_k, fmt, block, renormalize, out=out.view.view_as(x))
    out.check()
    want, bound = pu.moe64(pu.to64(x), lg, up[2], down[2], inner, top_k, renormalize, x.dtype)
    pu.check(got, want, bound)
    return got


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1", "int8", "int4"])
@pytest.mark.parametrize("t,e,top_k,hidden,inner,block", [(1, 1, 1, 32, 32, 32), (1, 8, 2, 256, 384, 128), (2, 5, 3, 96, 160, 32), (7, 9, 2, 192, 64, 64),
                                                         (32, 40, 4, 128, 96, 32), (64, 3, 3, 64, 128, 64)])
def test_moe(t, e, top_k, hidden, inner, block, fmt, dtype):
    rng = rng_of(t, e, top_k, hidden, inner)
    run_moe(*moe_case(rng, t, e, hidden, inner, fmt, block, dtype), inner, top_k, fmt, block)


@pytest.mark.parametrize("renormalize", [True, False])
def test_moe_choice(renormalize):
    """Ties, masked experts, rows with one expert or none, rows with a NaN, all tokens at one expert, every expert chosen."""
    rng = rng_of(11, 12)
    t, e, hidden, inner = 24, 12, 64, 32
    x, lg, up, down = moe_case(rng, t, e, hidden, inner, "int8", 32, FP)
    lg[0] = 1.5                                             # all equal: the lowest indices
    lg[1] = [0.0, -0.0] * 6                                 # zeros of both signs are equal
    lg[2] = -np.inf                                         # nobody
    lg[3] = -np.inf
    lg[3, 7] = -200.0                                       # one expert, fewer than top_k
    lg[4, 5] = np.nan
    lg[5:, 3] = 30.0                                        # more than eight tokens of one expert
    lg[6, :] = np.float32(np.finfo(np.float32).min)         # masked with the lowest value instead of -inf
    lg[6, 9] = 0.0
    lg[7, 0] = np.finfo(np.float32).max
    got = run_moe(x, lg, up, down, inner, 3, "int8", 32, renormalize)
    assert not got[2].any() and got[4].isnan().all()
    run_moe(x[:4], lg[:4], up, down, inner, e, "int8", 32, renormalize)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1", "int8", "int4"])
def test_moe_scales_at_the_ends_of_their_range(fmt):
    """Up matrices with scales far above one BF16 factor, met by small tokens; down matrices far below; a poisoned block of an expert
    that is not chosen, and one of an expert that is."""
    rng = rng_of(31, 7)
    t, e, hidden, inner, block = 5, 4, 128, 64, 32
    x, lg, up, down = moe_case(rng, t, e, hidden, inner, fmt, block, FP)
    lg[:, 3] = -np.inf
    us = up[1].cpu().numpy().astype(np.int64).reshape(e, -1)
    ds = down[1].cpu().numpy().astype(np.int64).reshape(e, -1)
    us[:] = np.clip(us + 100, 0, 254)
    ds[:] = np.clip(ds - 60, 0, 254)
    us[3, 5] = 255
    x = x * 2.0 ** -100

    def pair(got, s, rows, k):
        codes = orc.unpack(got[0].cpu().numpy(), e * rows * k, orc.bits(fmt)).astype(np.int64).reshape(e, rows, k)
        return got[0], dev(s.astype(np.uint8)), pu.values64(codes, s.reshape(e, rows, -1), fmt, block)

    u, d = pair(up, us, 2 * inner, hidden), pair(down, ds, hidden, inner)
    u[2][3] = 0.0                                           # the expert that nobody chooses
    run_moe(x, lg, u, d, inner, 2, fmt, block)
    lg[1] = [5.0, 0.0, 0.0, -np.inf]
    ds[0, 0] = 255                                          # row 0 of expert 0's down matrix
    d = pair(down, ds, hidden, inner)
    got = mxq.moe(x, dev(lg), u[0], u[1], d[0], d[1], inner, 2, fmt, block)
    chosen = [[c[0] for c in row] for row in pu.choice64(lg, 2, True)]
    for i in range(t):
        assert bool(got[i, 0].isnan()) == (0 in chosen[i])
        assert not got[i, 1:].isnan().any()


def test_moe_without_any_choice():
    rng = rng_of(47, 7)
    x, lg, up, down = moe_case(rng, 3, 5, 64, 32, "int8", 32, BF)
    got = mxq.moe(x, torch.full((3, 5), -float("inf"), device="cuda"), up[0], up[1], down[0], down[1], 32, 2, "int8", out=torch.full_like(x, 9))
    assert not got.any()
    assert mxq.moe(x[:0], dev(lg[:0]), up[0], up[1], down[0], down[1], 32, 2, "int8").shape == (0, 64)


def test_moe_takes_rows_of_a_larger_batch():
    """Tokens and logits that are views into a batch, the logits at any row."""
    rng = rng_of(43, 7)
    x, lg, up, down = moe_case(rng, 7, 5, 64, 32, "e4m3", 32, BF)
    lg = dev(lg)
    want = mxq.moe(x, lg, up[0], up[1], down[0], down[1], 32, 2, "e4m3")
    for i in range(7):
        assert torch.equal(mxq.moe(x[i:i + 1], lg[i:i + 1], up[0], up[1], down[0], down[1], 32, 2, "e4m3"), want[i:i + 1])


def test_moe_infinite_tokens_stay_in_their_rows():
    rng = rng_of(41, 7)
    x, lg, up, down = moe_case(rng, 4, 3, 64, 32, "e4m3", 32, BF)
    clean = mxq.moe(x, dev(lg), up[0], up[1], down[0], down[1], 32, 2, "e4m3")
    x[1, 3], x[2, 5] = float("inf"), float("nan")
    got = mxq.moe(x, dev(lg), up[0], up[1], down[0], down[1], 32, 2, "e4m3")
    assert torch.equal(got[0], clean[0]) and torch.equal(got[3], clean[3])
    assert not got[1].isfinite().any() and got[2].isnan().all()


def test_moe_offsets_beyond_32_bits():
    e, hidden, inner, block = 33, 8192, 8192, 128           # the up matrices pass 2^32 codes
    rng = rng_of(51, 7)
    used, rows = 32, 32
    x = torch.zeros(1, hidden, device="cuda")
    x[0, -rows:] = torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()
    up = torch.zeros(e * 2 * inner * hidden, dtype=torch.uint8, device="cuda")
    us = torch.full((up.numel() // block,), 127, dtype=torch.uint8, device="cuda")
    down = torch.zeros(e * hidden * inner, dtype=torch.uint8, device="cuda")
    ds = torch.full((down.numel() // block,), 127, dtype=torch.uint8, device="cuda")
    lg = torch.full((1, e), -float("inf"), device="cuda")
    lg[0, used] = 1.0
    u, d = up.view(e, 2 * inner, hidden), down.view(e, hidden, inner)
    code = torch.randint(0x20, 0x40, (3, rows), device="cuda", dtype=torch.uint8)
    u[used, inner - 1, -rows:], u[used, 2 * inner - 1, -rows:], d[used, -rows:, -1] = code[0], code[1], code[2]
    got = mxq.moe(x, lg, up, us, down, ds, inner, 1, "e4m3", block)
    v = pu.value_table("e4m3")[code.cpu().numpy()]
    xv = pu.to64(x)[0, -rows:]
    g, l = v[0] @ xv, v[1] @ xv
    h = g / (1 + np.exp(-g)) * l
    assert not got[:, :-rows].any()
    off = np.abs(v[0]) @ np.abs(xv) * (np.abs(l) + 1) + np.abs(v[1]) @ np.abs(xv) * np.abs(g) + np.abs(h)
    pu.check(got[0, -rows:], v[2] * h, pu.sum_bound(hidden, v[2] * off))


def test_moe_streams_graphs_and_workspaces():
    rng = rng_of(61, 7)
    t, e, hidden, inner = 6, 10, 128, 96
    x, lg, up, down = moe_case(rng, t, e, hidden, inner, "e2m1", 32, BF)
    lg, w = dev(lg), (up[0], up[1], down[0], down[1])
    want = mxq.moe(x, lg, *w, inner, 3, "e2m1")
    for _ in range(5):                                      # nothing is left in a workspace that a later call would see
        assert torch.equal(mxq.moe(x, lg, *w, inner, 3, "e2m1"), want)
    dirty = torch.full((mxq.moe_workspace_bytes(t, 3, inner),), 0xFF, dtype=torch.uint8, device="cuda")
    assert torch.equal(mxq.moe(x, lg, *w, inner, 3, "e2m1", workspace=dirty), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [mxq.moe(x, lg, *w, inner, 3, "e2m1", stream=s) for _ in range(3)]
    here = [mxq.moe(x, lg, *w, inner, 3, "e2m1") for _ in range(3)]       # at the same time, workspaces of their own
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in got + here)
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        outs.append(torch.empty_like(x))
        with torch.cuda.graph(graphs[-1]):
            mxq.moe(x, lg, *w, inner, 3, "e2m1", out=outs[-1])
    for k in range(4):
        outs[0].zero_()
        outs[1].zero_()
        with torch.cuda.stream(s):
            graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


# ---- together, as they are used -------------------------------------------------------------------------------


def test_train_a_linear_then_serve_its_codes():
    """Steps of a linear layer on quantized operands, then the trained weight's anchor in a product: the forward pass's bits."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(200, 96, generator=g, device="cuda", dtype=BF)
    target = torch.randn(200, 160, generator=g, device="cuda", dtype=BF)
    w = (torch.randn(160, 96, generator=g, device="cuda") * 0.05).requires_grad_()
    for _ in range(3):
        y = mxq.linear_ste(x, w, 32)
        loss = (y.float() - target.float()).square().mean()
        (dw,) = torch.autograd.grad(loss, w)
        assert dw.dtype == FP and dw.isfinite().all() and dw.any()
        with torch.no_grad():
            w -= 0.1 * dw
    y = mxq.linear_ste(x, w, 32).detach()
    wc, ws = mxq.quantize(w.detach(), "e4m3", 32)
    xc, xs = mxq.quantize(x, "e4m3", 32)
    assert torch.equal(mxq.matmul(xc, xs, wc, ws, 200, 160, 96, block=32), y)


def test_one_anchor_served_in_two_precisions_by_moe():
    """Experts stored as an E4M3 anchor, lowered to E2M1 by Slice-and-Scale, and the layer run on both."""
    rng = rng_of(71, 7)
    t, e, hidden, inner = 5, 6, 128, 64
    x, lg, up, down = moe_case(rng, t, e, hidden, inner, "e4m3", 32, BF)
    run_moe(x, lg, up, down, inner, 2, "e4m3", 32)
    low = []
    for got, rows, k in ((up, 2 * inner, hidden), (down, hidden, inner)):
        n = e * rows * k
        c, s = mxq.slice_scale(got[0], got[1], n, "e4m3", "e2m1")
        v = mxq.dequantize(c, s, n, "e2m1")
        low.append((c, s, pu.to64(v).reshape(e, rows, k)))
    run_moe(x, lg, low[0], low[1], inner, 2, "e2m1", 32)
