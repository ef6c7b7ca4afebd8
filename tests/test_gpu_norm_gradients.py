"""The kernel's gradients of the norm against central differences of the forward formula, along directions in which a
missing or wrong term shows."""
import numpy as np
import pytest
import torch

import mx_util as mx
from paper_2607_18631_amd import moe
from paper_2607_18631_amd.workloads import f32_to_bf16_bits
from test_gpu_add_rmsnorm import EPS, dev, forward64, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [(7, 352), (40, 2048), (9, 7168), (3, 16416)])
def test_against_differences(rows, d):
    """Row by row <dx, v> along h and at random, and <dgamma, v> along gamma and at random.  dy has a part along h, so the
    term of the mean is of order 1.  The results are bf16, each off by at most 2^-8 of itself, independently: a sum of
    such errors has a standard deviation below 2^-8 / sqrt(3) of the 2-norm of its terms, and 8 of those are taken.  The
    float32 sums before (2^-15 of the terms' 1-norm at most) come on top."""
    rng = np.random.default_rng(d)
    h = mx.bf16_values(f32_to_bf16_bits((rng.standard_normal((rows, d)) * 2.0 ** rng.integers(-2, 3, (rows, 1))).astype(np.float32)))
    gamma = mx.bf16_values(f32_to_bf16_bits((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)))
    rstd = 1 / np.sqrt((h * h).mean(1, keepdims=True) + EPS)
    dy = mx.bf16_values(f32_to_bf16_bits((rng.standard_normal((rows, d)) + rng.uniform(0.5, 2, (rows, 1)) * h * rstd).astype(np.float32)))
    dh = mx.bf16_values(f32_to_bf16_bits(rng.standard_normal((rows, d)).astype(np.float32)))
    bits = lambda v: dev(f32_to_bf16_bits(v.astype(np.float32)))
    x, g = bits(h), bits(gamma)
    y, r, dx, dgamma = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(g)
    moe.moe_add_rmsnorm(x, None, g, EPS, None, y, rstd=r)
    moe.moe_add_rmsnorm_backward(bits(dy), bits(dh), x, g, r, dx, dgamma, moe.alloc_add_rmsnorm_workspace(rows, d))
    dx, dgamma = host(dx), host(dgamma)
    loss = lambda h, g: (dy * forward64(h, g, EPS)[0]).sum(1) + (dh * h).sum(1)

    def check(terms, diff):
        tol = 8 * 2.0 ** -8 / np.sqrt(3) * np.linalg.norm(terms, axis=-1) + 2.0 ** -15 * np.abs(terms).sum(-1)
        assert (np.abs(terms.sum(-1) - diff) <= tol).all(), (np.abs(terms.sum(-1) - diff) / tol).max()
        return tol

    e = 1e-4
    for v in (h, rng.standard_normal((rows, d)) * np.linalg.norm(h, axis=1, keepdims=True) / np.sqrt(d)):
        tol = check(dx * v, (loss(h + e * v, gamma) - loss(h - e * v, gamma)) / (2 * e))
    # what leaving out the mean would change along h is far past that
    u, c = h * rstd, (dy * gamma * h * rstd).mean(1, keepdims=True)
    assert (np.abs((rstd * u * c * h).sum(1)) > 4 * tol).all()
    for v in (gamma, rng.standard_normal(d)):
        check(dgamma * v, ((loss(h, gamma + e * v) - loss(h, gamma - e * v)) / (2 * e)).sum())
