"""moe_add_rmsnorm and its backward on the GPU against float64."""
import numpy as np
import pytest
import torch

import mx_util as mx
from paper_2607_18631_amd import moe
from paper_2607_18631_amd.workloads import f32_to_bf16_bits

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
EPS = 1e-5
# a row of one vector, vectors that no wave divides, the edges between the kernels' row lengths, rows past a
# workgroup's registers
WIDTHS = [8, 24, 32, 504, 512, 520, 1024, 1056, 2040, 2048, 2080, 4096, 4104, 7168, 8192, 8224, 16384, 16416, 40968]


def bits(rng, *shape, std=1.0):
    return f32_to_bf16_bits((rng.standard_normal(shape) * std).astype(np.float32))


def dev(b):
    return moe.to_device_bf16(b)


def host(t):
    return t.double().cpu().numpy()


def forward64(h, gamma, eps):
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * gamma, rstd


def close(got, want, abs_part):
    """One rounding to bf16 (2^-8 of the value at most) on top of float32 errors: 2^-15 of the terms' size allows
    for 2^8 roundings of 2^-24 each and a sum's own."""
    err = np.abs(got - want)
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * abs_part
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), (worst, got[worst], want[worst])


def run_forward(rows, d, *, residual=True, y=True, q=False, rstd=True, alias=None, eps=EPS, seed=0, std=1.0):
    rng = np.random.default_rng(seed + d + rows)
    xb, rb, gb = bits(rng, rows, d, std=std), bits(rng, rows, d, std=2 * std), f32_to_bf16_bits(
        (1 + 0.2 * rng.standard_normal(d)).astype(np.float32))
    x, r, gamma = dev(xb), dev(rb) if residual else None, dev(gb)
    h = None if not residual else {"x": x, "residual": r, None: torch.empty_like(x)}[alias]
    # one row more than the call may write
    out = torch.full((rows + 1, d), -3.0, dtype=BF16, device="cuda")
    yq = torch.full((rows + 1, d), 0x11, dtype=torch.uint8, device="cuda") if q else None
    ys = torch.full((rows + 1, d // 32), 0x11, dtype=torch.uint8, device="cuda") if q else None
    rs = torch.full((rows + 1,), -3.0, device="cuda") if rstd else None
    moe.moe_add_rmsnorm(x, r, gamma, eps, h, out[:rows] if y else None, yq[:rows] if q else None,
                        ys[:rows] if q else None, rs[:rows] if rstd else None)
    xv, rv, gv = mx.bf16_values(xb), mx.bf16_values(rb), mx.bf16_values(gb)
    hv = xv
    if residual:
        # the sum is taken in float32, then rounded
        hv = mx.bf16_values(f32_to_bf16_bits(xv.astype(np.float32) + rv.astype(np.float32)))
        np.testing.assert_array_equal(host(h), hv)
    want, want_rstd = forward64(hv, gv, eps)
    if rstd:
        np.testing.assert_allclose(host(rs[:rows]), want_rstd, rtol=2.0 ** -18)
        assert rs[rows] == -3.0
    if y:
        close(host(out[:rows]), want, np.abs(want))
        assert (out[rows] == -3.0).all()
    if q:
        assert (yq[rows] == 0x11).all() and (ys[rows] == 0x11).all()
        got = yq[:rows].cpu().numpy(), ys[:rows].cpu().numpy()
        if y:
            codes, scales = mx.quantize(host(out[:rows]), mx.E4M3)
            np.testing.assert_array_equal(got[0], codes)
            np.testing.assert_array_equal(got[1], scales)
        return got
    return out[:rows]


@pytest.mark.parametrize("d", WIDTHS)
def test_forward_widths(d):
    for rows in (1, 3, 6):
        run_forward(rows, d, q=d % 32 == 0)


@pytest.mark.parametrize("rows", [1, 2, 4, 5, 255, 1030])
def test_forward_rows(rows):
    run_forward(rows, 736, q=True)


@pytest.mark.parametrize("d", [64, 2048, 7168, 16416])
def test_forward_options(d):
    """Without a residual, one result of two, no statistics, h in the buffer of x or of the residual: the same values."""
    whole = run_forward(5, d, q=True)
    only = run_forward(5, d, y=False, q=True, rstd=False)
    assert all(np.array_equal(a, b) for a, b in zip(whole, only))
    assert all(np.array_equal(a, b) for a, b in zip(whole, run_forward(5, d, q=True, alias="x")))
    assert all(np.array_equal(a, b) for a, b in zip(whole, run_forward(5, d, q=True, alias="residual")))
    run_forward(5, d, residual=False)
    run_forward(5, d, residual=False, q=True)


@pytest.mark.parametrize("rows,d", [(40000, 64), (3000, 2048), (2000, 7168), (200, 16416)])
def test_every_value_is_the_float64_one(rows, d):
    """The float64 result to float32 to bf16, in every bit: the 8-bit form's scale turns on the last."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, r = (torch.empty((rows, d), device="cuda").normal_(generator=g).to(BF16) for _ in range(2))
    gamma = (torch.empty(d, device="cuda").normal_(generator=g) * 0.3 + 1).to(BF16)
    h, y = torch.empty_like(x), torch.empty_like(x)
    moe.moe_add_rmsnorm(x, r, gamma, 1e-5, h, y)
    want = h.double() / (h.double().pow(2).mean(1, keepdim=True) + float(np.float32(1e-5))).sqrt() * gamma.double()
    assert torch.equal(y, want.float().to(BF16))


@pytest.mark.parametrize("d", [64, 2048, 7168, 16416])
def test_rows_of_no_finite_values_stay_alone(d):
    """Forward and backward: a NaN or an infinity reaches its own row's results and, backward, dgamma."""
    g = torch.Generator(device="cuda").manual_seed(d)
    x, r, dy = (torch.empty((9, d), device="cuda").normal_(generator=g).to(BF16) for _ in range(3))
    gamma = torch.ones(d, dtype=BF16, device="cuda")

    def run():
        h, y, dx, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty(9, device="cuda")
        q, s = torch.empty((9, d), dtype=torch.uint8, device="cuda"), torch.empty((9, d // 32), dtype=torch.uint8, device="cuda")
        dg = torch.empty_like(gamma)
        moe.moe_add_rmsnorm(x, r, gamma, 1e-6, h, y, q, s, rstd)
        moe.moe_add_rmsnorm_backward(dy, None, h, gamma, rstd, dx, dg, moe.alloc_add_rmsnorm_workspace(9, d))
        return y, q, s, rstd, dx

    good = run()
    x[2, d - 1], x[6, 0] = float("nan"), float("inf")
    got = run()
    others = torch.tensor([0, 1, 3, 4, 5, 7, 8], device="cuda")
    assert all(torch.equal(a[others], b[others]) for a, b in zip(got, good))
    assert torch.isnan(got[0][2]).all() and (got[2][2] == 255).all() and torch.isnan(got[4][2]).all()
    # an infinite row: rstd is 0, so its finite values give 0 and the infinite one NaN
    assert got[3][6] == 0 and (got[0][6, 1:] == 0).all() and torch.isnan(got[0][6, 0])


def test_more_rows_than_a_launch_has_threads_for():
    """2^28 + 3 rows of 8 values: offsets past 32 bits, and eight launches and a rest; every row against the formula in
    float64, in pieces."""
    rows, d, eps = (1 << 28) + 3, 8, 1e-5
    g = torch.Generator(device="cuda").manual_seed(4)
    x, y = torch.empty((rows, d), dtype=BF16, device="cuda"), torch.full((rows + 1, d), -3.0, dtype=BF16, device="cuda")
    for a in range(0, rows, 1 << 24):
        x[a:a + (1 << 24)].normal_(generator=g)
    gamma = torch.randn(d, generator=torch.Generator().manual_seed(5)).to(BF16).cuda()
    moe.moe_add_rmsnorm(x, None, gamma, eps, None, y[:rows])
    for a in range(0, rows, 1 << 24):
        b = min(rows, a + (1 << 24))
        h = x[a:b].double()
        ref = h / (h.pow(2).mean(1, keepdim=True) + eps).sqrt() * gamma.double()
        # half a step of bf16 and the statistics' float32 error
        assert ((y[a:b].double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -18) * ref.abs()).all(), a
    assert (y[rows] == -3.0).all()


def test_forward_scales_and_eps():
    for std in (1e-18, 1e-4, 1e4, 1e15):
        run_forward(4, 1088, std=std, eps=0.0)
        run_forward(4, 1088, std=std, eps=1.0)
    # rows of zeros are zeros with any eps above 0
    x = torch.zeros((3, 64), dtype=BF16, device="cuda")
    y, g = torch.full_like(x, 5.0), torch.ones(64, dtype=BF16, device="cuda")
    q, s = torch.ones((3, 64), dtype=torch.uint8, device="cuda"), torch.ones((3, 2), dtype=torch.uint8, device="cuda")
    moe.moe_add_rmsnorm(x, None, g, 1e-6, None, y, q, s)
    assert (y == 0).all() and (q == 0).all() and (s == 0).all()


def backward64(dy, dh, h, gamma, rstd):
    u = h * rstd[:, None]
    g = dy * gamma
    c = (g * u).mean(1, keepdims=True)
    dx = rstd[:, None] * (g - u * c) + (0 if dh is None else dh)
    return dx, (dy * u).sum(0)


def run_backward(rows, d, *, dh=True, alias=None, seed=0):
    rng = np.random.default_rng(seed + 3 * d + rows)
    hb, yb, rb = bits(rng, rows, d), bits(rng, rows, d), bits(rng, rows, d)
    gb = f32_to_bf16_bits((1 + 0.2 * rng.standard_normal(d)).astype(np.float32))
    hv, yv, rv, gv = map(mx.bf16_values, (hb, yb, rb, gb))
    rstd = (1 / np.sqrt((hv * hv).mean(1) + EPS)).astype(np.float32)
    dy, dh_t = dev(yb), dev(rb) if dh else None
    guard = torch.full((rows + 1, d), -3.0, dtype=BF16, device="cuda")
    dx = {"dy": dy, "dh": dh_t, None: guard[:rows]}[alias]
    dgamma = torch.full((d + 8,), -3.0, dtype=BF16, device="cuda")
    ws = moe.alloc_add_rmsnorm_workspace(rows, d)
    moe.moe_add_rmsnorm_backward(dy, dh_t, dev(hb), dev(gb), torch.from_numpy(rstd).cuda(), dx, dgamma[:d], ws)
    want_dx, want_dg = backward64(yv, rv if dh else None, hv, gv, rstd.astype(np.float64))
    u, g = np.abs(hv * rstd[:, None]), np.abs(yv * gv)
    close(host(dx), want_dx, rstd[:, None] * (g + u * (g * u).mean(1, keepdims=True)) + (np.abs(rv) if dh else 0))
    close(host(dgamma[:d]), want_dg, (np.abs(yv) * u).sum(0))
    assert (dgamma[d:] == -3.0).all() and (alias or (guard[rows] == -3.0).all())
    return dx.clone(), dgamma[:d].clone()


@pytest.mark.parametrize("d", WIDTHS)
def test_backward_widths(d):
    for rows in (1, 5, 37):
        run_backward(rows, d, dh=rows != 5)


@pytest.mark.parametrize("rows", [1, 2, 16, 17, 1000, 16395])
def test_backward_rows(rows):
    """Fewer rows than workgroups have, and more than one round of all workgroups."""
    run_backward(rows, 264)


@pytest.mark.parametrize("rows,d", [(1, 2056), (2, 2056), (3, 2056), (255, 2056), (257, 4104), (4100, 2056), (3, 16416), (300, 16416)])
def test_backward_long_rows(rows, d):
    """One workgroup, a workgroup per row, and several rows each."""
    run_backward(rows, d)


def test_backward_in_place_and_repeatable():
    for d in (512, 7168):
        a = run_backward(300, d)
        for alias in (None, "dy", "dh"):
            b = run_backward(300, d, alias=alias)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), alias


def test_backward_without_rows_clears_dgamma():
    e = torch.empty((0, 64), dtype=BF16, device="cuda")
    dgamma = torch.full((64,), 4.0, dtype=BF16, device="cuda")
    moe.moe_add_rmsnorm_backward(e, None, e, torch.ones(64, dtype=BF16, device="cuda"), torch.empty(0, device="cuda"), e,
                                 dgamma, moe.alloc_add_rmsnorm_workspace(0, 64))
    assert (dgamma == 0).all()


def test_gradients_against_differences():
    """<dx, v> and <dgamma, v> against central differences of sum(dy * y) + sum(dh * h), in float64, at the kernel's h.
    The differences' own error is below 1e-6; the kernel's results are bf16: 2^-8 of each term of the products."""
    rng = np.random.default_rng(4)
    rows, d = 7, 352
    hb, yb, rb = bits(rng, rows, d), bits(rng, rows, d), bits(rng, rows, d)
    gb = f32_to_bf16_bits((1 + 0.2 * rng.standard_normal(d)).astype(np.float32))
    hv, yv, rv, gv = map(mx.bf16_values, (hb, yb, rb, gb))
    x, gamma = dev(hb), dev(gb)
    y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    moe.moe_add_rmsnorm(x, None, gamma, EPS, None, y, rstd=rstd)
    dx, dgamma = torch.empty_like(x), torch.empty_like(gamma)
    moe.moe_add_rmsnorm_backward(dev(yb), dev(rb), x, gamma, rstd, dx, dgamma, moe.alloc_add_rmsnorm_workspace(rows, d))

    def loss(h, g):
        return (yv * forward64(h, g, EPS)[0]).sum() + (rv * h).sum()

    for grad, at in ((host(dx), 0), (host(dgamma), 1)):
        v = rng.standard_normal(grad.shape)
        e = 1e-5
        hi = loss(*((hv + e * v, gv) if at == 0 else (hv, gv + e * v)))
        lo = loss(*((hv - e * v, gv) if at == 0 else (hv, gv - e * v)))
        diff = (hi - lo) / (2 * e)
        assert abs((grad * v).sum() - diff) <= 2.0 ** -8 * np.abs(grad * v).sum() + 1e-5 * abs(diff)


def test_training_step_replays_in_a_graph():
    rng = np.random.default_rng(6)
    rows, d = 50, 1032
    x, r, dy, dh = (torch.zeros((rows, d), dtype=BF16, device="cuda") for _ in range(4))
    gamma = dev(f32_to_bf16_bits((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)))

    def buffers():
        e = torch.empty_like(x)
        return [torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), e, torch.empty_like(gamma),
                moe.alloc_add_rmsnorm_workspace(rows, d)]

    def step(b):
        moe.moe_add_rmsnorm(x, r, gamma, EPS, b[0], b[1], rstd=b[2])
        moe.moe_add_rmsnorm_backward(dy, dh, b[0], gamma, b[2], b[3], b[4], b[5])

    mine, eager = buffers(), buffers()
    step(mine)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(mine)
    for i in range(4):
        for t in (x, r, dy, dh):
            t.copy_(dev(bits(rng, rows, d)))
        graph.replay()
        got = [t.clone() for t in mine[:5]]
        step(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), i
