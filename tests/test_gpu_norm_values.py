"""moe_add_rmsnorm on rows at the ends of bf16's range: every y is the bf16 of the float32 of the float64 formula, and the
8-bit form is y's."""
import numpy as np
import pytest
import torch

import mx_util as mx
from paper_2607_18631_amd import moe

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def rows_of(seed, rows, d, low, high):
    """Signed bf16 rows of magnitudes spread evenly between two bounds."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = torch.rand((rows, d), device="cuda", generator=g, dtype=torch.float64) * (high - low) + low
    sign = torch.randint(0, 2, (rows, d), device="cuda", generator=g) * 2 - 1
    return (m * sign).to(BF16)


def check(x, gamma, eps):
    rows, d = x.shape
    y, q, s = torch.empty_like(x), torch.empty((rows, d), dtype=torch.uint8, device="cuda"), torch.empty(
        (rows, d // 32), dtype=torch.uint8, device="cuda")
    moe.moe_add_rmsnorm(x, None, gamma, eps, None, y, q, s)
    h = x.double()
    want = h / (h.pow(2).mean(1, keepdim=True) + float(np.float32(eps))).sqrt() * gamma.double()
    want = want.float().to(BF16)
    assert torch.equal(y, want), ((y != want).sum().item(), y[y != want][:4], want[y != want][:4])
    codes, scales = mx.quantize(want.double().cpu().numpy(), mx.E4M3)
    np.testing.assert_array_equal(q.cpu().numpy(), codes)
    np.testing.assert_array_equal(s.cpu().numpy(), scales)
    return y


@pytest.mark.parametrize("d", [64, 2048, 7168, 16416])
def test_large_rows(d):
    """Magnitudes from 1.5e38 to bf16's largest: h * gamma is past float32, h * rstd * gamma about 1 to 4."""
    x = rows_of(d, 64, d, 1.5e38, 3.3e38)
    for seed, (low, high) in enumerate(((2.5, 4.0), (100.0, 200.0))):
        assert torch.isfinite(check(x, rows_of(seed, 1, d, low, high)[0], 1e-5)).all()


@pytest.mark.parametrize("d", [64, 2048, 7168, 16416])
def test_small_rows_without_eps(d):
    """eps = 0: rows whose product with gamma is subnormal in float32, and rows of bf16's subnormal numbers, whose rstd is
    past float32."""
    assert torch.isfinite(check(rows_of(d, 64, d, 1e-37, 8e-36), rows_of(3, 1, d, 1e-5, 1e-3)[0], 0.0)).all()
    y = check(rows_of(d + 1, 64, d, 1e-40, 3e-39), rows_of(4, 1, d, 0.5, 2.0)[0], 0.0)
    assert torch.isfinite(y).all() and (y.abs() > 1e-3).all()


@pytest.mark.parametrize("d", [64, 7168])
def test_large_gamma(d):
    """Values whose product with rstd alone is subnormal in float32."""
    x = rows_of(d, 64, d, 0.5, 2.0)
    x[:, ::3] = rows_of(d + 1, 64, d, 1e-38, 1e-36)[:, ::3]
    x[:, 1] = 3e4
    check(x, rows_of(5, 1, d, 1e28, 1e30)[0], 0.0)
