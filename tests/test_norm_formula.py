"""The gradient formula that the GPU tests of the norm compare with, against central differences in float64 (no GPU),
and that differences find the mistakes such a formula can have."""
import numpy as np
import pytest

from test_gpu_add_rmsnorm import EPS, backward64, forward64

ROWS, D, STEP = 7, 352, 1e-4


def case(eps=EPS, seed=4):
    """Rows of several sizes, and dy with a part along h, so that the mean of g u is of order 1."""
    rng = np.random.default_rng(seed)
    h = rng.standard_normal((ROWS, D)) * 2.0 ** np.arange(-3, 4)[:, None]
    gamma = 1 + 0.2 * rng.standard_normal(D)
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    dy = rng.standard_normal((ROWS, D)) + rng.uniform(0.5, 2, (ROWS, 1)) * h * rstd[:, None]
    return h, gamma, rstd, dy, rng.standard_normal((ROWS, D))


def worst(formula, eps):
    """Largest error of <gradient, v> over the row's (or dgamma's) |gradient| |v|, for directions along each row, and at
    random."""
    h, gamma, rstd, dy, dh = case(eps)
    dx, dgamma = formula(dy, dh, h, gamma, rstd)
    rng = np.random.default_rng(1)
    loss = lambda h, g: (dy * forward64(h, g, eps)[0]).sum(1) + (dh * h).sum(1)
    errors = []
    for v in (h / np.linalg.norm(h, axis=1, keepdims=True), rng.standard_normal((ROWS, D)), rng.standard_normal((ROWS, D))):
        e = STEP * np.linalg.norm(h, axis=1, keepdims=True) / np.linalg.norm(v, axis=1, keepdims=True) * v
        diff = (loss(h + e, gamma) - loss(h - e, gamma)) / 2
        size = np.linalg.norm(dx, axis=1) * np.linalg.norm(e, axis=1)
        errors.append(np.max(np.abs((dx * e).sum(1) - diff) / size))
    for v in (gamma, rng.standard_normal(D)):
        e = STEP * v
        diff = (loss(h, gamma + e) - loss(h, gamma - e)).sum() / 2
        errors.append(abs((dgamma * e).sum() - diff) / (np.linalg.norm(dgamma) * np.linalg.norm(e)))
    return max(errors)


# A step of 1e-4 of the row: the third-order term is about STEP^2 = 1e-8 of the first, the roundings of the two losses
# (2^-53 of sums of some 10^3) over the step some 1e-9 of it.
TOL = 1e-6


@pytest.mark.parametrize("eps", [EPS, 0.5])
def test_formula_against_differences(eps):
    assert worst(backward64, eps) <= TOL


MISTAKES = {
    "no mean": lambda r, g, u, c: r * g,
    "mean of the other sign": lambda r, g, u, c: r * (g + u * c),
    "no outer rstd": lambda r, g, u, c: g - u * c,
    "sum over one value more": lambda r, g, u, c: r * (g - u * c * D / (D + 1)),
    "rstd twice": lambda r, g, u, c: r * (g - u * r * c),
}


@pytest.mark.parametrize("name", MISTAKES)
def test_differences_find_a_mistake_in_dx(name):
    def formula(dy, dh, h, gamma, rstd):
        r, g, u = rstd[:, None], dy * gamma, h * rstd[:, None]
        return MISTAKES[name](r, g, u, (g * u).mean(1, keepdims=True)) + dh, (dy * u).sum(0)
    assert worst(formula, EPS) > 100 * TOL


def test_differences_find_a_missing_dh_and_a_wrong_dgamma():
    assert worst(lambda dy, dh, h, g, r: (backward64(dy, None, h, g, r)[0], backward64(dy, dh, h, g, r)[1]), EPS) > 100 * TOL
    assert worst(lambda dy, dh, h, g, r: (backward64(dy, dh, h, g, r)[0], (dy * h).sum(0)), EPS) > 100 * TOL
