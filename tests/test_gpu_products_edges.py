"""The operators that multiply by stored codes where the values, addresses and derivatives are unusual: against their definitions in
64 bits (product_util)."""
import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq
import paper_2604_00529_b200.binding  # noqa: F401
import torch.utils.checkpoint  # noqa: F401

import product_util as pu

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- E4M3's NaN codes -----------------------------------------------------------------------------------------


def e4m3_values(codes, scales, block):
    """Values in 64 bits, S.1111.111 a NaN."""
    v = pu.values64(codes.astype(np.int64), scales.astype(np.int64), "e4m3", block)
    return np.where((codes & 0x7F) == 0x7F, np.nan, v)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_moe_weights_that_are_nan_codes(dtype):
    """One token per expert, one NaN code in most experts: at each of a lane's 16 places, of either sign, in up or in down matrices.  A NaN
    in an up matrix makes all of the token NaN, one in a down matrix the element of its row; every other code is a number."""
    rng = np.random.default_rng(5)
    t, e, hidden, inner, block = 40, 41, 256, 64, 32
    up = rng.integers(0, 256, (e, 2 * inner, hidden)).astype(np.uint8)
    down = rng.integers(0, 256, (e, hidden, inner)).astype(np.uint8)
    up[(up & 0x7F) == 0x7F] ^= 1                            # all codes, the NaN codes aside
    down[(down & 0x7F) == 0x7F] ^= 1
    for i in range(16):
        up[i, (37 * i) % (2 * inner), 16 * ((5 * i) % 16) + i] = 0x7F | (i & 1) << 7
        down[16 + i, (53 * i) % hidden, 16 * (i % 4) + i] = 0x7F | (~i & 1) << 7
    up[40], down[40] = 0x7F, 0xFF                           # the expert that nobody chooses
    us = rng.integers(110, 118, (e, 2 * inner, hidden // block)).astype(np.uint8)
    ds = rng.integers(110, 118, (e, hidden, inner // block)).astype(np.uint8)
    x = torch.from_numpy(rng.standard_normal((t, hidden)).astype(np.float32)).cuda().to(dtype)
    lg = np.full((t, e), -np.inf, np.float32)
    lg[np.arange(t), np.arange(t)] = 1.0
    got = mxq.moe(x, dev(lg), dev(up), dev(us), dev(down), dev(ds), inner, 1, "e4m3", block)
    want, bound = pu.moe64(pu.to64(x), lg, e4m3_values(up, us, block), e4m3_values(down, ds, block), inner, 1, True, dtype)
    assert np.isnan(want[:16]).all() and (np.isnan(want[16:32]).sum(1) == 1).all() and not np.isnan(want[32:]).any()
    pu.check(got, want, bound)


@pytest.mark.parametrize("m", [2, 40, 300])
def test_matmul_operands_that_are_nan_codes(m):
    rng = np.random.default_rng(m)
    n, k, block = 130, 256, 64
    a, b = (rng.integers(0, 256, (r, k)).astype(np.uint8) for r in (m, n))
    for c in (a, b):
        c[(c & 0x7F) == 0x7F] ^= 1
    a[m // 2, 77], b[n // 3, 200] = 0x7F, 0xFF
    sa, sb = (rng.integers(110, 118, (r, k // block)).astype(np.uint8) for r in (m, n))
    av, bv = e4m3_values(a, sa, block), e4m3_values(b, sb, block)
    got = mxq.matmul(dev(a), dev(sa), dev(b), dev(sb), m, n, k, block=block, dtype=FP)
    pu.check(got, av @ bv.T, pu.sum_bound(k, np.abs(av) @ np.abs(bv).T))


# ---- linear_ste -----------------------------------------------------------------------------------------------


@pytest.fixture(params=[True, False], ids=["native", "general"])
def path(request, monkeypatch):
    """Both ways a linear_ste call can go: the binding's native code, and the Python code behind it."""
    if not request.param:
        mxq.load_library()
        monkeypatch.setattr(mxq.binding._host, "linear_ste", lambda *a: None)


def offset_copy(t, elements):
    """t's values in a contiguous view that begins `elements` elements into its storage."""
    flat = torch.empty(t.numel() + elements, device=t.device, dtype=t.dtype)
    v = flat[elements:].view(t.shape)
    v.copy_(t)
    assert v.is_contiguous() and v.data_ptr() % 32
    return v


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m,n,k", [(9, 33, 37), (40, 64, 96)])
def test_linear_ste_at_any_address(path, m, n, k, dtype):
    """Operands and gradients that are contiguous at addresses of no particular alignment: the bits of the aligned ones."""
    g = torch.Generator(device="cuda").manual_seed(m)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(dtype) for s in ((m, k), (n, k), (m, n)))
    xa, wa = x.clone().requires_grad_(), w.clone().requires_grad_()
    want = mxq.linear_ste(xa, wa)
    want = [want.detach(), *torch.autograd.grad(want, (xa, wa), dy)]
    for off in ((1, 0, 0), (0, 3, 0), (0, 0, 1), (5, 7, 3)):
        xo, wo, go = (offset_copy(t, o) if o else t.clone() for t, o in zip((x, w, dy), off))
        xo.requires_grad_(), wo.requires_grad_()
        y = mxq.linear_ste(xo, wo)
        for a, b in zip([y.detach(), *torch.autograd.grad(y, (xo, wo), go)], want):
            assert torch.equal(a, b)


def test_linear_ste_of_slices_and_joined_outputs(path):
    """x[1:] of an odd width, a weight inside a flat parameter buffer, outputs joined by cat: the gradients arrive as views at offsets."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(8, 37, generator=g, device="cuda", dtype=BF)
    flat = torch.randn(1 + 1000 * 37, generator=g, device="cuda").to(BF).requires_grad_()
    w = flat[1:].view(1000, 37)
    dy = torch.randn(7 + 333, 1000, generator=g, device="cuda").to(BF)
    other = torch.randn(333, 37, generator=g, device="cuda", dtype=BF)
    joined = torch.cat((mxq.linear_ste(other, w), mxq.linear_ste(x[1:], w)))
    (got,) = torch.autograd.grad(joined, flat, dy)
    w2 = flat.detach()[1:].clone().view(1000, 37).requires_grad_()
    y1, y2 = mxq.linear_ste(other, w2), mxq.linear_ste(x[1:].clone(), w2)
    assert torch.equal(joined, torch.cat((y1, y2)))
    (want,) = torch.autograd.grad((y1, y2), w2, (dy[:333].clone(), dy[333:].clone()))
    assert torch.equal(got[1:].view(1000, 37), want) and got[0] == 0


@pytest.mark.parametrize("shape,n", [((5, 0), 3), ((0,), 4), ((2, 3, 0), 5), ((0, 0), 3), ((4, 7), 0), ((2, 0, 7), 0)])
def test_linear_ste_without_any_products(path, shape, n):
    """Empty sums are zeros; empty results have their shapes."""
    x = torch.randn(shape, device="cuda", requires_grad=True)
    w = torch.randn(n, shape[-1], device="cuda", requires_grad=True)
    y = mxq.linear_ste(x, w)
    assert y.shape == (*shape[:-1], n) and not y.any()
    dx, dw = torch.autograd.grad(y, (x, w), torch.ones_like(y))
    assert dx.shape == x.shape and dw.shape == w.shape and not dx.any() and not dw.any()


def test_linear_ste_gradients_refuse_to_be_differentiated(path):
    """Also where the incoming gradient is a constant: dx depends on w and dw on x all the same."""
    x = torch.randn(4, 32, device="cuda", requires_grad=True)
    w = torch.randn(8, 32, device="cuda", requires_grad=True)
    plain = torch.autograd.grad(mxq.linear_ste(x, w).sum(), (x, w))
    for loss in (lambda y: y.sum(), lambda y: y.square().sum()):
        for leaves in ((x,), (w,), (x, w)):
            y = mxq.linear_ste(x, w)
            grads = torch.autograd.grad(loss(y), leaves, create_graph=True)
            penalty = sum(g.square().sum() for g in grads)
            with pytest.raises(RuntimeError, match="differentiated once"):
                (loss(y) + penalty).backward()
    x.grad = w.grad = None
    mxq.linear_ste(x, w).sum().backward(create_graph=True)     # gradients that nobody differentiates are the usual ones
    assert torch.equal(x.grad, plain[0]) and torch.equal(w.grad, plain[1])
    with pytest.raises(RuntimeError, match="differentiated once"):
        x.grad.square().sum().backward()
    x.grad, w.grad = x.grad.detach(), w.grad.detach()
    mxq.linear_ste(x, w).sum().backward()
    assert torch.equal(x.grad, 2 * plain[0]) and torch.equal(w.grad, 2 * plain[1])
    assert not any(g.requires_grad for g in torch.autograd.grad(mxq.linear_ste(x, w).sum(), (x, w)))


# ---- streams --------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("handle", [0, 1, 2])
def test_streams_given_as_the_fixed_handles(handle):
    """The default stream, cudaStreamLegacy and cudaStreamPerThread."""
    x = torch.randn(96, 160, device="cuda")
    want = mxq.quantize_matrix(x)
    torch.cuda.synchronize()
    got = mxq.quantize_matrix(x, stream=handle)
    d = mxq.matmul(got[0], got[1], got[0], got[1], 96, 96, 160, stream=handle)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(d, mxq.matmul(*want[:2], *want[:2], 96, 96, 160))


# ---- linear_ste inside the rest of torch ----------------------------------------------------------------------


def test_linear_ste_refuses_transforms(path):
    """vmap, the functional derivatives and forward-mode derivatives raise; nothing is answered silently."""
    x, w = torch.randn(4, 32, device="cuda"), torch.randn(8, 32, device="cuda")
    for call in (lambda: torch.func.vmap(lambda t: mxq.linear_ste(t, w))(x[None]),
                 lambda: torch.func.vmap(lambda t: t * mxq.linear_ste(x, w).sum())(x),
                 lambda: torch.func.grad(lambda t: mxq.linear_ste(t, w).sum())(x),
                 lambda: torch.func.jvp(lambda t: mxq.linear_ste(t, w), (x,), (x,))):
        with pytest.raises(RuntimeError):
            call()
    with torch.autograd.forward_ad.dual_level(), pytest.raises(RuntimeError):
        mxq.linear_ste(torch.autograd.forward_ad.make_dual(x, x), w)


def test_linear_ste_traced_hooked_and_recomputed(path):
    g = torch.Generator(device="cuda").manual_seed(9)
    x, w = torch.randn(4, 32, generator=g, device="cuda"), torch.randn(8, 32, generator=g, device="cuda")
    traced = torch.jit.trace(lambda t: mxq.linear_ste(t, w), (x,), check_trace=False)
    other = torch.randn(6, 32, generator=g, device="cuda")
    assert torch.equal(traced(other), mxq.linear_ste(other, w))
    xr, wr = x.clone().requires_grad_(), w.clone().requires_grad_()
    want = torch.autograd.grad(mxq.linear_ste(xr, wr), (xr, wr), torch.full((4, 8), 2.0, device="cuda"))
    seen = []
    y = mxq.linear_ste(xr, wr)
    y.register_hook(lambda t: 2 * t)
    handle = xr.register_hook(lambda t: seen.append(t.shape))
    y.sum().backward()
    handle.remove()
    assert seen == [xr.shape] and torch.equal(xr.grad, want[0]) and torch.equal(wr.grad, want[1])
    y = torch.utils.checkpoint.checkpoint(mxq.linear_ste, xr, wr, use_reentrant=False)
    for a, b in zip(torch.autograd.grad(2 * y.sum(), (xr, wr)), want):
        assert torch.equal(a, b)
    y = mxq.linear_ste(xr, wr)                              # twice through one graph, where it was kept
    first = torch.autograd.grad(2 * y.sum(), (xr, wr), retain_graph=True)
    for a, b, c in zip(first, torch.autograd.grad(2 * y.sum(), (xr, wr)), want):
        assert torch.equal(a, c) and torch.equal(b, c)


def test_moe_has_no_gradient():
    x = torch.randn(2, 64, device="cuda", requires_grad=True)
    up, down = mxq.quantize(torch.randn(4 * 64 * 64, device="cuda"), "int8"), mxq.quantize(torch.randn(4 * 64 * 32, device="cuda"), "int8")
    got = mxq.moe(x, torch.randn(2, 4, device="cuda"), *up, *down, 32, 2, "int8")
    assert not got.requires_grad and got.isfinite().all()
