"""The checks of precision_util have teeth: results with fewer bits than promised fail them, sums in 32 bits pass."""
import numpy as np
import pytest
import torch

import precision_util as pr


@pytest.mark.parametrize("k", [4096, 14336])
def test_norm_limit_tells_32_bits_from_fewer(k):
    g = torch.Generator().manual_seed(k)
    a, b = torch.randn(40, k, generator=g).bfloat16(), torch.randn(30, k, generator=g).bfloat16()
    want = a.double() @ b.double().t()
    near, cut = torch.zeros(40, 30), torch.zeros(40, 30)
    for i in range(0, k, 32):                               # a step's products exactly, with the sum so far rounded, or cut, to FP32
        step = a[:, i:i + 32].double() @ b[:, i:i + 32].double().t()
        near = (near.double() + step).float()
        exact = cut.double() + step
        cut = exact.float()
        cut = torch.where(cut.double().abs() > exact.abs(), torch.nextafter(cut, torch.zeros(())), cut)
    assert pr.norm_error(near, want) <= pr.norm_limit(k) / 10
    assert pr.norm_limit(k) / 10 <= pr.norm_error(cut, want) <= pr.norm_limit(k)
    assert pr.norm_error(want.bfloat16(), want) > 30 * pr.norm_limit(k)
    parts = [a[:, i::4].double() @ b[:, i::4].double().t() for i in range(4)]
    assert pr.norm_error(sum(v.bfloat16().double() for v in parts).float(), want) > 30 * pr.norm_limit(k)
    assert pr.norm_error(sum(v.half().double() for v in parts).float(), want) > 3 * pr.norm_limit(k)


@pytest.mark.parametrize("fmt", pr.FORMATS)
def test_one_product_tells_three_parts_from_two(fmt):
    x, lg, *_, up, down = pr.one_product(np.random.default_rng(3), fmt)
    want, bound = pr.one_product64(x, lg, up, down)
    assert np.abs(want).max() > 0.1 and (want != 0).mean() > 0.5
    same, _ = pr.one_product64(x, lg, up, down, lambda v: pr.bf16_parts(v, 3), lambda v: pr.bf16_parts(v, 3))
    assert (np.abs(same - want) <= bound).all()             # all 24 bits: FP32's rounding of h alone
    fewer, _ = pr.one_product64(x, lg, up, down, keep_x=lambda v: pr.bf16_parts(v, 2))
    assert (np.abs(fewer - want) > bound).mean() > 0.1
    fewer, _ = pr.one_product64(x, lg, up, down, keep_h=lambda v: pr.bf16_parts(v, 2))
    assert (np.abs(fewer - want) > bound).mean() > 0.1
