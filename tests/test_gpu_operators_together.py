"""The operators as a program uses them one after another: norm, routing, permutation, conversion, expert MLP
and combine of a prefill step; a few tokens through a stack of norms and layers, captured; a training step of norm and
layer and both their gradients.  Each against float64."""
import numpy as np
import pytest
import torch

import mx_util as mx
import oracle
import parity_util as pu
from oracle import moe_backward as obwd
from paper_2607_18631_amd import moe
from paper_2607_18631_amd import workloads as wl
from paper_2607_18631_amd.workloads import MoEShape

pytestmark = pytest.mark.gpu
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
EPS = 1e-6


def empty(*shape, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def f64(t):
    return t.double().cpu().numpy()


def normal(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(BF16).cuda()


def norm64(h, gamma):
    rstd = 1 / np.sqrt((h ** 2).mean(-1, keepdims=True) + EPS)
    return h * rstd * gamma, rstd


def check_norm(h, y, x, residual, gamma):
    """h is the float32 sum rounded once; y is within half a step of bf16, and the statistics' float32 error."""
    assert torch.equal(h, (x.float() + residual.float()).to(BF16))
    ref = norm64(f64(h), f64(gamma))[0]
    assert (np.abs(f64(y) - ref) <= (2.0 ** -8 + 2.0 ** -18) * np.abs(ref)).all()


class Experts:
    """e2m1 weights of a layer on the GPU, and their float64 values."""

    def __init__(self, sh, seed):
        self.sh = sh
        for name, rows, K in (("w13", sh.E_local * 2 * sh.F, sh.d), ("w2", sh.E_local * sh.d, sh.F),
                              ("ws13", 2 * sh.F_shared, sh.d), ("ws2", sh.d, sh.F_shared)):
            seed += 1
            q = s = v = None
            if rows and K:
                q, s, w = empty(rows, K // 2, dtype=U8), empty(rows, K // 32, dtype=U8), empty(rows, K)
                moe.moe_mx_quantize(moe.MOE_MX_E2M1, normal(seed, rows, K, scale=K ** -0.5), q, s)
                moe.moe_mx_dequantize(moe.MOE_MX_E2M1, q, s, w)         # exact: 2 significant bits
                v = f64(w)
            setattr(self, name, q), setattr(self, name + "_scales", s), setattr(self, name + "_values", v)

    def mlp(self, e, x, round_activation):
        F = self.sh.F
        w = self.w13_values[e * 2 * F:(e + 1) * 2 * F]
        a, b = x @ w[:F].T, x @ w[F:].T
        return round_activation(a / (1 + np.exp(-a)) * b) @ self.w2_values[e * self.sh.d:(e + 1) * self.sh.d].T


@pytest.mark.parametrize("fmt", [moe.MOE_MX_E2M1, moe.MOE_MX_E4M3])
@pytest.mark.parametrize("sh", [
    MoEShape(T=48, d=256, E=16, top_k=4, F=96, E_local=16),
    MoEShape(T=301, d=544, E=24, top_k=3, F=160, E_local=8, e_begin=8),     # a slice: some slots have no row
    MoEShape(T=60, d=128, E=8, top_k=2, F=64, E_local=8, expert_capacity=12),   # slots past the capacity are dropped
], ids=["all", "slice", "capacity"])
def test_prefill_step(sh, fmt):
    w = Experts(sh, 100)
    gamma, w_router = normal(1, sh.d, scale=0.2) + 1, normal(2, sh.E, sh.d, scale=sh.d ** -0.5)
    x, residual, h, y = normal(3, sh.T, sh.d), normal(4, sh.T, sh.d), empty(sh.T, sh.d), empty(sh.T, sh.d)
    idx, gates = empty(sh.T, sh.top_k, dtype=I32), empty(sh.T, sh.top_k, dtype=F32)
    counts, offsets = empty(sh.E_local, dtype=I32), empty(sh.E_local + 1, dtype=I32)
    cap = sh.capacity
    row_token, slot_row = empty(cap, dtype=I32), empty(sh.T, sh.top_k, dtype=I32)
    # rows that no slot fills keep what a new buffer holds; it may be anything, here NaN
    x_perm = torch.full((cap, sh.d), float("nan"), dtype=BF16, device="cuda")
    q, s = empty(cap, moe.mx_elements_per_row(fmt, sh.d), dtype=U8), empty(cap, sh.d // 32, dtype=U8)
    ws = {k: moe.alloc_workspace(sh, k) for k in (moe.MOE_WS_ROUTE, moe.MOE_WS_PERMUTE, moe.MOE_WS_MX_FFN)}

    def step(y_perm, out):
        moe.moe_add_rmsnorm(x, residual, gamma, EPS, h, y)
        moe.moe_route(sh, y, w_router, None, idx, gates, None, ws[moe.MOE_WS_ROUTE])
        moe.moe_permute(sh, idx, y, counts, offsets, row_token, slot_row, x_perm, ws[moe.MOE_WS_PERMUTE])
        moe.moe_mx_quantize(fmt, x_perm, q, s)
        moe.moe_mx_grouped_ffn(sh, fmt, q, s, counts if sh.expert_capacity else offsets, w.w13, w.w13_scales, w.w2,
                               w.w2_scales, y_perm, ws[moe.MOE_WS_MX_FFN])
        moe.moe_combine(sh, y_perm, slot_row, gates, None, out)

    y_perm, out = torch.full_like(x_perm, 5.0), torch.full_like(x, 9.0)
    step(y_perm, out)
    check_norm(h, y, x, residual, gamma)
    rows = mx.rounded(f64(y), fmt)
    chosen, gate, ref = idx.cpu().numpy(), f64(gates), np.zeros((sh.T, sh.d))
    for e in range(sh.E_local):
        tok, slot = np.nonzero(chosen == sh.e_begin + e)
        if sh.expert_capacity:
            tok, slot = tok[:sh.expert_capacity], slot[:sh.expert_capacity]
        if len(tok):
            ref[tok] += gate[tok, slot][:, None] * w.mlp(e, rows[tok], lambda a: mx.rounded(a, fmt))
    # the expert rows' own tolerance (5e-3 of the norm: two roundings and the activation's rounding borders) and the
    # result's rounding
    assert pu.rel_fro(f64(out), ref) <= 5e-3 + 2.0 ** -8
    live = slot_row.cpu().numpy()
    untouched = np.ones(cap, bool)
    untouched[live[live >= 0]] = False
    assert (f64(y_perm)[untouched] == 5.0).all()

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(y_perm, out)
    for i in range(4):
        x.copy_(normal(50 + i, sh.T, sh.d))
        graph.replay()
        torch.cuda.synchronize()
        got, eager = out.clone(), torch.empty_like(out)
        step(torch.empty_like(y_perm), eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), i


@pytest.mark.parametrize("T", [1, 5, 40])
def test_few_tokens_through_a_stack(T):
    """Three layers with a workspace between them: h += layer(norm(h)), eager, as one graph and as a graph per layer."""
    sh = MoEShape(T=T, d=256, E=16, top_k=4, F=96, E_local=16, F_shared=64)
    layers = [(Experts(sh, 10 * i), normal(200 + i, sh.E, sh.d, scale=sh.d ** -0.5), normal(300 + i, sh.d, scale=0.2) + 1)
              for i in range(3)]
    x, h, y, out = normal(1, T, sh.d), empty(T, sh.d), empty(T, sh.d), empty(T, sh.d)
    ws = moe.alloc_workspace(sh, moe.MOE_WS_DECODE)
    n = T * sh.top_k

    def layer(i):
        w, w_router, gamma = layers[i]
        # the stream is h itself from the second layer on, updated in place
        moe.moe_add_rmsnorm(out if i else x, h if i else zero, gamma, EPS, h, y)
        moe.moe_layer_decode(sh, y, w_router, None, w.w13, w.w2, w.ws13, w.ws2, out, ws,
                             (w.w13_scales, w.w2_scales, w.ws13_scales, w.ws2_scales))

    zero = torch.zeros_like(h)
    for i in range(3):
        before, add = (h.clone(), out.clone()) if i else (zero, x)
        layer(i)
        check_norm(h, y, add, before, layers[i][2])
        w, w_router = layers[i][:2]
        chosen, gate = ws[:4 * n].view(I32).view(T, -1).cpu().numpy(), None
        at = moe.workspace_offset(sh, moe.MOE_REGION_TOPK_W)
        gate = f64(ws[at:at + 4 * n].view(F32).view(T, -1))
        L = f64(y) @ f64(w_router).T
        keys = oracle.gating_keys(L, sh.gate, None)
        top = np.sort(L, 1)[:, ::-1]
        if (top[:, sh.top_k - 1] - top[:, sh.top_k] > 2.0 ** -18 * np.abs(L).max()).all():
            assert np.array_equal(np.sort(chosen, 1), np.sort(oracle.decide_topk(keys, sh.top_k, 1, 1), 1))
        np.testing.assert_allclose(gate, oracle.gate_weights(keys, chosen, sh.gate, sh.renormalize, 1.0), rtol=0, atol=1e-5)
        ref = np.zeros((T, sh.d))
        half = lambda a: f64(torch.from_numpy(a).float().to(BF16))         # the activation is bf16
        for t in range(T):
            for j, e in enumerate(chosen[t]):
                ref[t] += gate[t, j] * w.mlp(e, f64(y)[t:t + 1], half)[0]
        Fs, a = sh.F_shared, f64(y) @ w.ws13_values.T
        ref += half(a[:, :Fs] / (1 + np.exp(-a[:, :Fs])) * a[:, Fs:]) @ w.ws2_values.T
        assert pu.rel_fro(f64(out), ref) <= pu.REL_TOL

    eager = out.clone()
    whole, parts = torch.cuda.CUDAGraph(), [torch.cuda.CUDAGraph() for _ in layers]
    with torch.cuda.graph(whole):
        for i in range(3):
            layer(i)
    for i, g in enumerate(parts):
        with torch.cuda.graph(g):
            layer(i)
    for k in range(4):
        x.copy_(normal(60 + k, T, sh.d))
        for i in range(3):
            layer(i)
        eager = out.clone()
        torch.cuda.synchronize()
        whole.replay()
        assert torch.equal(out, eager), k
        out.zero_()
        for g in parts:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager), k


def test_training_step_of_norm_and_layer():
    """h = x + r, out = h + layer(norm(h)): gradients of x and gamma through both backward passes."""
    sh = MoEShape(T=96, d=264, E=16, top_k=4, F=96, E_local=16)
    inputs = wl.custom_inputs(sh, seed=31)
    layer = moe.DeviceLayer(inputs)
    x, residual, gamma = normal(5, sh.T, sh.d), normal(6, sh.T, sh.d), normal(7, sh.d, scale=0.2) + 1
    dout = normal(8, sh.T, sh.d)
    h, y, rstd = empty(sh.T, sh.d), empty(sh.T, sh.d), empty(sh.T, dtype=F32)
    moe.moe_add_rmsnorm(x, residual, gamma, EPS, h, y, rstd=rstd)
    check_norm(h, y, x, residual, gamma)
    layer.x = y
    layer.forward()
    dy = layer.backward(dout)["dx"]
    dx, dgamma = empty(sh.T, sh.d), empty(sh.d)
    moe.moe_add_rmsnorm_backward(dy, dout, h, gamma, rstd, dx, dgamma, moe.alloc_add_rmsnorm_workspace(sh.T, sh.d))
    torch.cuda.synchronize()

    idx, w, keys = pu.run_route(layer)
    layer_in = dict(inputs, x=pu.dev_bits(y))
    o_idx, o_w, keys64, near = pu.check_routing(layer_in, idx, w, keys)
    routing = pu.oracle_routing_with_gpu_ties(o_idx, o_w, keys64, idx, near, sh)
    dy64 = obwd.layer_backward(layer_in, f64(dout), routing=routing)["dx"]
    h64, g64 = f64(h), f64(gamma)
    _, r = norm64(h64, g64)
    u, g = h64 * r, dy64 * g64
    dx64 = r * (g - u * (g * u).mean(-1, keepdims=True)) + f64(dout)
    dg64 = (dy64 * u).sum(0)
    # dy's error (REL_TOL of its norm) passes through a projection times rstd and gamma; dx is rounded once more
    most = (r * np.abs(g64)).max()
    assert np.linalg.norm(f64(dx) - dx64) <= most * pu.REL_TOL * np.linalg.norm(dy64) + 2.0 ** -8 * np.linalg.norm(dx64)
    # each column's sum: at most |error of dy's column| * |u's column|
    col = np.linalg.norm(f64(dy) - dy64, axis=0) * np.linalg.norm(u, axis=0)
    assert (np.abs(f64(dgamma) - dg64) <= col + 2.0 ** -7 * np.abs(dg64) + 1e-5 * np.abs(dy64 * u).sum(0)).all()
    assert np.linalg.norm(f64(dy) - dy64) <= pu.REL_TOL * np.linalg.norm(dy64)


def test_two_streams_at_once():
    """The same weights and different rows on two streams, each with its own buffers; and again in turn."""
    sh = MoEShape(T=600, d=512, E=8, top_k=1, F=256, E_local=8)
    w = Experts(sh, 400)
    offsets = torch.tensor([0, 10, 10, 300, 301, 430, 500, 555, 600], dtype=I32, device="cuda")
    x = [normal(70 + i, sh.T, sh.d) for i in range(2)]
    gamma = normal(1, sh.d, scale=0.2) + 1

    def run(i, out):
        y, q, s = empty(sh.T, sh.d), empty(sh.T, sh.d, dtype=U8), empty(sh.T, sh.d // 32, dtype=U8)
        moe.moe_add_rmsnorm(x[i], None, gamma, EPS, None, y, q, s)
        moe.moe_mx_grouped_ffn(sh, moe.MOE_MX_E4M3, q, s, offsets, w.w13, w.w13_scales, w.w2, w.w2_scales, out,
                               moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN))

    alone = [empty(sh.T, sh.d) for _ in x]
    for i in range(2):
        run(i, alone[i])
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in x], [empty(sh.T, sh.d) for _ in x]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                run(i, both[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(both[i], alone[i])
