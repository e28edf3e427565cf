"""FP32 results of the products are as exact as sums in 32 bits are (limits and inputs: precision_util)."""
import numpy as np
import pytest
import torch

import paper_2604_00529_b200 as mxq

import precision_util as pr
import product_util as pu

pytestmark = pytest.mark.gpu
FP = torch.float32


def operand(g, rows, k, block):
    """Random finite E4M3 codes and scale bytes, and their values in 64 bits."""
    codes = torch.randint(0, 256, (rows, k), generator=g, device="cuda", dtype=torch.uint8)
    codes = torch.where((codes & 0x7F) == 0x7F, codes ^ 1, codes)
    scales = torch.randint(118, 122, (rows, k // block), generator=g, device="cuda", dtype=torch.uint8)
    values = torch.from_numpy(pu.value_table("e4m3")).cuda()[codes.long()]
    return codes, scales, values * torch.exp2(scales.double() - 127).repeat_interleave(block, 1)


@pytest.mark.parametrize("m,n,k,block", [(1, 128, 4096, 128), (8, 200, 4096, 64), (5, 96, 4096, 32), (13, 400, 14336, 128), (40, 2000, 14336, 32),
                                         (200, 512, 14336, 64), (512, 4096, 14336, 128), (700, 4096, 14336, 128), (700, 4099, 14336, 32)])
def test_matmul_long_sums(m, n, k, block):
    """Every kind of launch: few rows, k in parts, CTA pairs with 128 and 256 columns."""
    g = torch.Generator(device="cuda").manual_seed(m)
    a, sa, av = operand(g, m, k, block)
    b, sb, bv = operand(g, n, k, block)
    err = pr.norm_error(mxq.matmul(a, sa, b, sb, m, n, k, block=block, dtype=FP), av @ bv.t())
    print("%d x %d x %d, blocks of %d: %.2g of %.2g" % (m, n, k, block, err, pr.norm_limit(k)))
    assert err <= pr.norm_limit(k)


def test_linear_ste_long_sums():
    """dw over 14336 rows of tokens, from the codes that the quantizer gives."""
    m, n, k, block = 14336, 96, 160, 32
    g = torch.Generator(device="cuda").manual_seed(7)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda") for s in ((m, k), (n, k), (m, n)))
    leaf = w.clone().requires_grad_()
    (dw,) = torch.autograd.grad(mxq.linear_ste(x, leaf, block), leaf, dy)

    def values(t):
        _, _, codes, scales = mxq.quantize_matrix(t, block=block, rows=False)
        v = torch.from_numpy(pu.value_table("e4m3")).cuda()[codes.long()].view(t.shape[1], m)
        return v * torch.exp2(scales.double() - 127).view(t.shape[1], -1).repeat_interleave(block, 1)

    err = pr.norm_error(dw, values(dy) @ values(x).t())
    print("%.2g of %.2g" % (err, pr.norm_limit(m)))
    assert err <= pr.norm_limit(m)


@pytest.mark.parametrize("fmt", pr.FORMATS)
def test_moe_keeps_all_bits_of_fp32_tokens(fmt):
    x, lg, uc, us, dc, ds, up, down = pr.one_product(np.random.default_rng(11), fmt)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    got = mxq.moe(dev(x), dev(lg), dev(uc), dev(us), dev(dc), dev(ds), down.shape[2], 1, fmt)
    want, bound = pr.one_product64(x, lg, up, down)
    worst = float((np.abs(pu.to64(got) - want) / bound).max())
    print("%s: %.2g of the bound" % (fmt, worst))
    assert worst <= 1.0


@pytest.mark.parametrize("fmt", pr.FORMATS)
def test_moe_long_sums(fmt):
    """A matrix step of the warp cuts its sum: 24 of them at most between two additions in FP32, 24 2^-23 2/3 = 1.9e-6 of the sum; the gate's
    and the up half's errors meet in h with a factor of 2.3 together, the down matrix adds its own: 6.3e-6, and the limit is 1e-5."""
    rng = np.random.default_rng(13)
    t, e, hidden, inner, block = 6, 4, 4096, 2048, 128
    x = torch.from_numpy(rng.standard_normal((t, hidden)).astype(np.float32)).cuda()
    lg = torch.from_numpy(rng.standard_normal((t, e)).astype(np.float32)).cuda()
    up, down = (mxq.quantize(torch.from_numpy((rng.standard_normal(n) * s).astype(np.float32)).cuda(), fmt, block)
                for n, s in ((e * 2 * inner * hidden, 0.02), (e * hidden * inner, 0.03)))
    got = mxq.moe(x, lg, *up, *down, inner, 2, fmt, block)
    u = mxq.dequantize(*up, e * 2 * inner * hidden, fmt, block).view(e, 2 * inner, hidden).double()
    d = mxq.dequantize(*down, e * hidden * inner, fmt, block).view(e, hidden, inner).double()
    gu = torch.einsum("erk,tk->ter", u, x.double())
    each = torch.einsum("ehi,tei->teh", d, torch.nn.functional.silu(gu[..., :inner]) * gu[..., inner:])
    top = torch.topk(lg.double(), 2, -1)
    want = (each.gather(1, top.indices[..., None].expand(-1, -1, hidden)) * top.values.softmax(-1)[..., None]).sum(1)
    err = pr.norm_error(got, want)
    print("%s: %.2g" % (fmt, err))
    assert err <= 1e-5
