"""8-bit products whose scales are far from 1."""
import pytest
import torch

import paper_2508_12851_amd as P
import i8_reference as R

pytestmark = pytest.mark.gpu

# every epilogue: low and high tiles, short contractions, contractions that are shared, stores through strips
SIZES = [(5, 64, 4096), (70, 131, 4096), (128, 128, 128), (300, 520, 384), (600, 4096, 2048), (2048, 8192, 512)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_scales_whose_product_is_not_a_normal_number(m, n, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(m)
    a, b = (torch.randint(64, 128, (r, k), generator=gen, device="cuda", dtype=torch.int8) for r in (m, n))
    sa = (1 + torch.rand(m, generator=gen, device="cuda")) * 2.0 ** -75
    sb = (1 + torch.rand(n, generator=gen, device="cuda")) * 2.0 ** -65
    got = P.prism_matmul_i8(P.prism_pack_i8(a, sa), P.prism_pack_i8(b, sb), P.alloc_matmul_i8_workspace(m, n, k), dtype=dtype)
    want = R.product(a.double(), sa.double(), b, sb)
    assert float((sa.max() * sb.max()).double()) < 2.0 ** -126 <= float(want.min())
    # no sum cancels, so that the roundings are relative to the result: the sum's, the two products', the addition of parts (7), the output's
    tol = 10 * R.EPS + (0 if dtype == torch.float32 else 2.0 ** -8 * (1 + 2.0 ** -8))
    assert bool(((got.double() - want).abs() <= tol * want).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_a_sum_of_zero_is_zero_whatever_the_scales(m, n, k, dtype):
    a = torch.ones((m, k), dtype=torch.int8, device="cuda")
    a[:, ::2] = -1
    b = torch.full((n, k), 100, dtype=torch.int8, device="cuda")
    sa, sb = torch.full((m,), 3e20, device="cuda"), torch.full((n,), 3e20, device="cuda")
    got = P.prism_matmul_i8(P.prism_pack_i8(a, sa), P.prism_pack_i8(b, sb), P.alloc_matmul_i8_workspace(m, n, k), dtype=dtype)
    assert int((got != 0).sum()) == 0
