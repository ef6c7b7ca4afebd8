"""Block-scaled formats on the GPU: conversion both ways bit for bit, and the grouped expert MLP on such
operands against float64."""
import numpy as np
import pytest
import torch

import mx_util as mx
import oracle
from paper_2607_18631_amd import moe
from paper_2607_18631_amd.workloads import MoEShape, f32_to_bf16_bits

pytestmark = pytest.mark.gpu
FORMATS = [mx.E2M1, mx.E4M3]
U8 = torch.uint8


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def quantize(bits, fmt, stream=None):
    """uint16 bf16 bits [rows, cols] through moe_mx_quantize -> (elements, scales) on the GPU."""
    x = moe.to_device_bf16(bits)
    rows, cols = bits.shape
    q = torch.full((rows, moe.mx_elements_per_row(fmt, cols)), 0xa5, dtype=U8, device="cuda")
    s = torch.full((rows, cols // 32), 0xa5, dtype=U8, device="cuda")
    moe.moe_mx_quantize(fmt, x, q, s, stream)
    return q, s


def check_quantize(bits, fmt):
    q, s = quantize(bits, fmt)
    codes, scales = mx.quantize(mx.bf16_values(bits), fmt)
    np.testing.assert_array_equal(s.cpu().numpy(), scales)
    np.testing.assert_array_equal(q.cpu().numpy(), mx.pack(codes, fmt))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 7168), (3, 96), (5, 2080), (67, 416), (1025, 64)])
def test_quantize_normal_rows(fmt, rows, cols):
    rng = np.random.default_rng(rows * 7919 + cols)
    check_quantize(f32_to_bf16_bits(rng.standard_normal((rows, cols)).astype(np.float32)), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_every_bf16_value(fmt):
    """Each of the 65536 bf16 patterns as the value beside a block maximum some exponents above it (the subnormal
    range, ties, cut values), and alone in its block; blocks with Inf or NaN among them."""
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    for up in (0, 1, 2, 3, 5, 9, 17):
        e = np.minimum((bits >> 7 & 255).astype(np.int64) + up, 254)
        blocks = np.zeros((65536, 32), np.uint16)
        blocks[:, 0] = (e << 7 | 0x7f) if up else 0
        blocks[:, 31] = bits
        check_quantize(blocks.reshape(-1, 1024), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_ties_and_zeros(fmt):
    """Every midpoint of the grid times every scale that bf16 reaches, zeros of both signs."""
    grid = mx.GRID[fmt]
    mid = (grid[1:] + grid[:-1]) / 2
    mid = np.concatenate([mid, -mid, [0.0, -0.0]])
    mid = np.resize(mid, (len(mid) + 30) // 31 * 31).reshape(-1, 31)
    for p in (-120, -30, 0, 1, 60, 110):
        rows = np.concatenate([np.full((len(mid), 1), grid[-1]), mid], 1) * 2.0 ** p
        bits = f32_to_bf16_bits(rows.astype(np.float32))
        assert np.array_equal(mx.bf16_values(bits), rows.astype(np.float32))
        check_quantize(bits, fmt)
    check_quantize(np.array([[0x0000, 0x8000] * 16] * 3, np.uint16), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_dequantize_every_code_and_scale(fmt):
    codes = np.tile(np.arange(16 if fmt == mx.E2M1 else 256, dtype=np.uint8), 2 if fmt == mx.E2M1 else 1)
    codes = np.tile(codes, (256, 1))                                     # [256 scales, 32 or 256]
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], codes.shape[1] // 32, 1)
    out = torch.empty(codes.shape, dtype=torch.bfloat16, device="cuda")
    moe.moe_mx_dequantize(fmt, dev(mx.pack(codes, fmt)), dev(scales), out)
    want = mx.round_bf16(mx.values(codes, scales, fmt))
    np.testing.assert_array_equal(out.double().cpu().numpy(), want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_dequantize_undoes_quantize(fmt):
    """What is on the grid already comes back as it is; rows of odd counts, guard rows stay."""
    rng = np.random.default_rng(5)
    for rows, cols in ((1, 32), (7, 352), (129, 4096)):
        q, s = quantize(f32_to_bf16_bits(rng.standard_normal((rows, cols)).astype(np.float32)), fmt)
        buf = torch.full((rows + 1, cols), 7.0, dtype=torch.bfloat16, device="cuda")
        moe.moe_mx_dequantize(fmt, q, s, buf[:rows])
        assert (buf[rows] == 7.0).all()
        q2, s2 = torch.empty_like(q), torch.empty_like(s)
        moe.moe_mx_quantize(fmt, buf[:rows], q2, s2)
        again = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
        moe.moe_mx_dequantize(fmt, q2, s2, again)
        assert torch.equal(again, buf[:rows])


@pytest.mark.parametrize("fmt", FORMATS)
def test_offsets_past_32_bits(fmt):
    """2^31 values and some rows: the last rows as alone, and back."""
    cols = 1024
    rows = (1 << 31) // cols + 5
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-9:].normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    q, s = torch.empty((rows, moe.mx_elements_per_row(fmt, cols)), dtype=U8, device="cuda"), torch.empty((rows, cols // 32), dtype=U8, device="cuda")
    moe.moe_mx_quantize(fmt, x, q, s)
    codes, scales = mx.quantize(x[-9:].double().cpu().numpy(), fmt)
    np.testing.assert_array_equal(s[-9:].cpu().numpy(), scales)
    np.testing.assert_array_equal(q[-9:].cpu().numpy(), mx.pack(codes, fmt))
    assert not q[:-9].any() and not s[:-9].any()
    moe.moe_mx_dequantize(fmt, q, s, x)
    np.testing.assert_array_equal(x[-9:].double().cpu().numpy(), mx.values(codes, scales, fmt))


# ---- expert MLP ----
def weights(rng, rows, K):
    """e2m1 weights of fan-in K: (elements, scales) on the GPU and their float64 values."""
    bits = f32_to_bf16_bits((rng.standard_normal((rows, K)) * K ** -0.5).astype(np.float32))
    codes, scales = mx.quantize(mx.bf16_values(bits), mx.E2M1)
    return dev(mx.pack(codes, mx.E2M1)), dev(scales), mx.values(codes, scales, mx.E2M1)


def mlp64(x, w13, w2, fmt):
    F = w2.shape[1]
    h, u = x @ w13[:F].T, x @ w13[F:].T
    return mx.rounded(h / (1 + np.exp(-h)) * u, fmt) @ w2.T


# Results are bf16 (each off by at most 2^-8 of its value, 1.7e-3 in the norm).  The float32 sums of the
# up-projection are off by some 1e-6 of their size, so about that share (over the grid's step, at least 2^-4 of the
# value) of the activations falls on the other side of a rounding border, each by one step: below
# sqrt(1e-4) * 2^-2 = 2.5e-3 of the norm.  Together below 5e-3.
REL = 5e-3


def run_mlp(fmt, d, F, counts, capacity=0, seed=0):
    """Runs the MLP on experts of `counts` rows; compares every live row, and that no other row was written."""
    rng = np.random.default_rng(seed)
    E = len(counts)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = E * capacity if capacity else max(1, int(offsets[-1]))
    sh = MoEShape(T=rows if not capacity else max(1, int(sum(counts))), d=d, E=E, top_k=1, F=F, E_local=E,
                  expert_capacity=capacity)
    assert sh.capacity == rows
    bits = f32_to_bf16_bits(rng.standard_normal((rows, d)).astype(np.float32))
    x_codes, x_scales = mx.quantize(mx.bf16_values(bits), fmt)
    live = np.zeros(rows, bool)
    segs = []
    for e in range(E):
        a = e * capacity if capacity else offsets[e]
        n = min(counts[e], capacity) if capacity else counts[e]
        segs.append((a, n))
        live[a:a + n] = True
    # rows outside every segment hold NaN scales: nothing of them may reach a result
    x_scales[~live] = 255
    w13, s13, v13 = weights(rng, E * 2 * F, d)
    w2, s2, v2 = weights(rng, E * d, F)
    y = torch.full((rows, d), -77.0, dtype=torch.bfloat16, device="cuda")
    ws = moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN)
    off = dev(np.asarray(counts, np.int32) if capacity else offsets)
    x_q, x_s = dev(mx.pack(x_codes, fmt)), dev(x_scales)
    moe.moe_mx_grouped_ffn(sh, fmt, x_q, x_s, off, w13, s13, w2, s2, y, ws)
    got = y.double().cpu().numpy()
    assert (got[~live] == -77.0).all()
    x = mx.values(x_codes, np.where(x_scales == 255, 0, x_scales), fmt)
    num = den = 0.0
    for e, (a, n) in enumerate(segs):
        if n:
            ref = mlp64(x[a:a + n], v13[e * 2 * F:(e + 1) * 2 * F], v2[e * d:(e + 1) * d], fmt)
            off2, size = np.sum((got[a:a + n] - ref) ** 2), np.sum(ref ** 2)
            assert np.sqrt(off2 / size) <= 2 * REL, f"expert {e}: {np.sqrt(off2 / size):.2e}"
            num, den = num + off2, den + size
    assert den > 0 and np.sqrt(num / den) <= REL, f"{np.sqrt(num / den):.2e}"
    return got


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,F", [(32, 32), (64, 96), (96, 160), (128, 128), (256, 288), (544, 224), (512, 1408)])
def test_mlp_widths(fmt, d, F):
    """K ends inside a slice, a block, and on it; output widths off the tiles."""
    run_mlp(fmt, d, F, [3, 0, 40, 1, 17])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,F", [(32, 64), (416, 224), (608, 736), (640, 1056), (1312, 544)])
def test_mlp_rows_whose_scales_start_at_any_byte(fmt, d, F):
    """Rows of 1 to 41 scales, so that they start at every byte of a word and end past every one; the rows around an
    expert's, in the equal-stride layout, have NaN scales, and so has every weight row of an expert without rows."""
    run_mlp(fmt, d, F, [3, 0, 70, 1, 17, 129])
    run_mlp(fmt, d, F, [2, 5, 0, 7], capacity=7, seed=1)
    run_mlp(fmt, d, F, [1])                                            # the tensors end with the row


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts", [[1], [0, 1, 0], [31, 32, 33], [64, 65, 127, 2], [130, 0, 128, 129, 1],
                                    [255, 256, 257], [600, 3, 0, 511]])
def test_mlp_rows(fmt, counts):
    run_mlp(fmt, 384, 256, counts, seed=len(counts))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,F", [(1024, 512), (1152, 640), (1056, 544)])
def test_mlp_enough_rows_to_fill_the_chip(fmt, d, F):
    """64 experts of 70 rows in the mean, from none to more than a tile of 256; K of whole slices of 256, of 128,
    and neither."""
    counts = [300, 257, 0, 1, 64, 65, 128, 129, 191, 192, 255, 256]
    counts += [(4480 - sum(counts)) // 52 + (i % 3 - 1) * 20 for i in range(52)]
    assert sum(counts) > 64 * 64
    run_mlp(fmt, d, F, counts, seed=d)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("capacity,counts", [(4, [0, 3, 4, 9]), (48, [48, 50, 1]), (160, [160, 7, 0, 159])])
def test_mlp_capacity_layout(fmt, capacity, counts):
    run_mlp(fmt, 256, 320, counts, capacity=capacity)


@pytest.mark.parametrize("fmt", FORMATS)
def test_mlp_many_experts(fmt):
    rng = np.random.default_rng(3)
    run_mlp(fmt, 64, 64, rng.integers(0, 4, 300).tolist())


@pytest.mark.parametrize("fmt", FORMATS)
def test_mlp_repeats_bit_for_bit(fmt):
    a, b = (run_mlp(fmt, 512, 384, [200, 31, 90], seed=11) for _ in range(2))
    assert np.array_equal(a, b)


@pytest.mark.parametrize("fmt", FORMATS)
def test_mlp_long_sums_keep_float32(fmt):
    """K = 7168 with products of one sign: the sum grows far past its terms."""
    d, F = 7168, 32
    sh = MoEShape(T=3, d=d, E=1, top_k=1, F=F, E_local=1)
    rng = np.random.default_rng(2)
    x = rng.choice([0.5, 1.0, 1.5, 3.0], (3, d)) * 2.0 ** -6
    w = rng.choice([0.5, 1.0, 2.0, 3.0], (2 * F, d)) * 2.0 ** -7
    xc, xs = mx.quantize(x, fmt)
    wc, wsc = mx.quantize(w, mx.E2M1)
    w2, s2, v2 = weights(rng, d, F)
    y = torch.empty((3, d), dtype=torch.bfloat16, device="cuda")
    moe.moe_mx_grouped_ffn(sh, fmt, dev(mx.pack(xc, fmt)), dev(xs), dev(np.array([0, 3], np.int32)),
                           dev(mx.pack(wc, mx.E2M1)), dev(wsc), w2, s2, y, moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN))
    ref = mlp64(mx.values(xc, xs, fmt), mx.values(wc, wsc, mx.E2M1), v2, fmt)
    assert np.linalg.norm(y.double().cpu().numpy() - ref) <= REL * np.linalg.norm(ref)


@pytest.mark.parametrize("fmt", FORMATS)
def test_mlp_offsets_past_32_bits(fmt):
    """Rows whose elements and results lie past 2^31 (values of the result, bytes of 8-bit rows): the last expert's 9
    rows against float64, the others' zeros."""
    d, F, before, n = 7168, 32, 300003, 9
    rows = before + n
    sh = MoEShape(T=rows, d=d, E=2, top_k=1, F=F, E_local=2)
    rng = np.random.default_rng(6)
    codes, scales = mx.quantize(mx.bf16_values(f32_to_bf16_bits(rng.standard_normal((n, d)).astype(np.float32))), fmt)
    q = torch.zeros((rows, moe.mx_elements_per_row(fmt, d)), dtype=U8, device="cuda")
    s = torch.full((rows, d // 32), 127, dtype=U8, device="cuda")
    q[before:], s[before:] = dev(mx.pack(codes, fmt)), dev(scales)
    w13, s13, v13 = weights(rng, 2 * 2 * F, d)
    w2, s2, v2 = weights(rng, 2 * d, F)
    y = torch.full((rows, d), -77.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mx_grouped_ffn(sh, fmt, q, s, dev(np.array([0, before, rows], np.int32)), w13, s13, w2, s2, y,
                           moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN))
    assert not y[:before].any()
    ref = mlp64(mx.values(codes, scales, fmt), v13[2 * F:], v2[d:], fmt)
    assert np.linalg.norm(y[before:].double().cpu().numpy() - ref) <= REL * np.linalg.norm(ref)


@pytest.mark.parametrize("fmt", FORMATS)
def test_mlp_rows_of_no_finite_values_stay_alone(fmt):
    """Rows that hold a NaN, an infinity, or e4m3's NaN code under a finite scale; and bf16's largest values, whose
    activation overflows: the other rows' results do not change by a bit."""
    d, F, n = 512, 96, 70
    sh = MoEShape(T=n, d=d, E=2, top_k=1, F=F, E_local=2)
    rng = np.random.default_rng(14)
    w13, s13, _ = weights(rng, 2 * 2 * F, d)
    w2, s2, _ = weights(rng, 2 * d, F)
    off = dev(np.array([0, 33, n], np.int32))
    x = moe.to_device_bf16(f32_to_bf16_bits(rng.standard_normal((n, d)).astype(np.float32)))
    ws = moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN)

    def run(code=False):
        q, s = torch.empty((n, moe.mx_elements_per_row(fmt, d)), dtype=U8, device="cuda"), torch.empty((n, d // 32), dtype=U8, device="cuda")
        moe.moe_mx_quantize(fmt, x, q, s)
        if code:
            q[40, 17] = 0x7f
        y = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
        moe.moe_mx_grouped_ffn(sh, fmt, q, s, off, w13, s13, w2, s2, y, ws)
        return y

    good = run()
    x[0, 5], x[31, 511], x[69] = float("nan"), float("inf"), 3.0e38
    bad = [0, 31, 69] + ([40] if fmt == mx.E4M3 else [])
    got = run(code=fmt == mx.E4M3)
    others = torch.ones(n, dtype=torch.bool, device="cuda")
    others[bad] = False
    assert torch.equal(got[others], good[others])
    for r in bad:
        assert not torch.isfinite(got[r]).any(), r


def test_mlp_replays_in_a_graph():
    """Captured conversion and MLP, replayed on new rows with eager work in between."""
    d, F, E = 256, 192, 4
    rng = np.random.default_rng(8)
    offsets = dev(np.array([0, 9, 9, 50, 64], np.int32))
    sh = MoEShape(T=64, d=d, E=E, top_k=1, F=F, E_local=E)
    w13, s13, _ = weights(rng, E * 2 * F, d)
    w2, s2, _ = weights(rng, E * d, F)
    x = torch.zeros((64, d), dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty((64, d), dtype=U8, device="cuda"), torch.empty((64, d // 32), dtype=U8, device="cuda")
    y, ws = torch.empty_like(x), moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN)

    def step(y, ws):
        moe.moe_mx_quantize(mx.E4M3, x, q, s)
        moe.moe_mx_grouped_ffn(sh, mx.E4M3, q, s, offsets, w13, s13, w2, s2, y, ws)

    step(y, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(y, ws)
    for i in range(4):
        x.copy_(moe.to_device_bf16(f32_to_bf16_bits(rng.standard_normal((64, d)).astype(np.float32))))
        graph.replay()
        got = y.clone()
        eager = torch.empty_like(y)
        step(eager, moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN))
        torch.cuda.synchronize()
        assert torch.equal(got, eager), i


def test_runs_on_the_stream_it_is_given():
    rng = np.random.default_rng(9)
    bits = f32_to_bf16_bits(rng.standard_normal((64, 512)).astype(np.float32))
    side = torch.cuda.Stream()
    x = torch.zeros((64, 512), dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty((64, 512), dtype=U8, device="cuda"), torch.empty((64, 16), dtype=U8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.copy_(moe.to_device_bf16(bits))
        moe.moe_mx_quantize(mx.E4M3, x, q, s)             # the current stream
    moe.moe_mx_quantize(mx.E4M3, x, q, s, side.cuda_stream)
    side.synchronize()
    codes, scales = mx.quantize(mx.bf16_values(bits), mx.E4M3)
    assert np.array_equal(q.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)
