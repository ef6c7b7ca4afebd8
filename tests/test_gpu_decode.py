"""moe_layer_decode on the GPU against the float64 oracle, with bf16 and with 4-bit weights."""
import numpy as np
import pytest
import torch

import mx_util as mx
import oracle
import parity_util as pu
from paper_2607_18631_amd import moe
from paper_2607_18631_amd import workloads as wl
from paper_2607_18631_amd.workloads import GATE_SIGMOID, MoEShape, f32_to_bf16_bits

pytestmark = pytest.mark.gpu
I32 = torch.int32


def make(shape, mixed, seed=0, zipf_s=0.0):
    """Workload inputs; with `mixed`, the expert weights are values of e2m1 blocks (exact in bf16, so the oracle
    reads them as the kernel does)."""
    inputs = wl.custom_inputs(shape, seed=seed, zipf_s=zipf_s)
    if mixed:
        for n in ("w13", "w2", "ws13", "ws2"):
            if inputs[n] is not None:
                v = mx.rounded(mx.bf16_values(inputs[n]), mx.E2M1)
                inputs[n] = f32_to_bf16_bits(v.astype(np.float32))
                assert np.array_equal(mx.bf16_values(inputs[n]), v)
    return inputs


def routing(layer):
    """(experts, gates) that the call left in its workspace."""
    sh, n = layer.shape, layer.shape.T * layer.shape.top_k
    off = [moe.workspace_offset(sh, r) for r in (moe.MOE_REGION_TOPK_IDX, moe.MOE_REGION_TOPK_W)]
    idx = layer.ws_decode[off[0]:off[0] + 4 * n].view(I32).view(sh.T, sh.top_k).cpu().numpy()
    w = layer.ws_decode[off[1]:off[1] + 4 * n].view(torch.float32).view(sh.T, sh.top_k).cpu().numpy()
    return idx, w


def reference(inputs, idx, w):
    """Output of the layer for given experts and gates, token by token."""
    sh = inputs["shape"]
    x = oracle.bf16_to_f64(inputs["x"])
    out = np.zeros((sh.T, sh.d))
    C = sh.expert_capacity
    for e in range(sh.E_local):
        tok, slot = np.nonzero(idx == sh.e_begin + e)
        if C > 0:
            tok, slot = tok[:C], slot[:C]
        if len(tok):
            y = oracle.swiglu_ffn(x[tok], oracle.bf16_to_f64(inputs["w13"][e]), oracle.bf16_to_f64(inputs["w2"][e]))
            out[tok] += w[tok, slot][:, None] * y
    if sh.F_shared:
        out += oracle.swiglu_ffn(x, oracle.bf16_to_f64(inputs["ws13"]), oracle.bf16_to_f64(inputs["ws2"]))
    return out


def check(shape, mixed, seed=0, zipf_s=0.0):
    inputs = make(shape, mixed, seed, zipf_s)
    layer = moe.DeviceLayer(inputs)
    if mixed:
        layer.quantize()
        layer.w13 = layer.w2 = layer.ws13 = layer.ws2 = None
    layer.out.fill_(99.0)
    got = layer.decode(mx=mixed).double().cpu().numpy()
    idx, w = routing(layer)
    # the decision is the float64 one except at rounding ties, the gates its gates
    sh = inputs["shape"]
    L = oracle.router_logits(oracle.bf16_to_f64(inputs["x"]), oracle.bf16_to_f64(inputs["w_router"]))
    keys = oracle.gating_keys(L, sh.gate, inputs.get("bias"))
    o_idx = oracle.decide_topk(keys, sh.top_k, sh.n_group, sh.topk_group)
    # float32 sums of d bf16 products, in up to 16 chunks of MFMA sums: 2^-18 of the logits' size is past their error
    kerr = 2.0 ** -18 * max(1.0, np.abs(L).max())
    for t in np.nonzero((o_idx != idx).any(1))[0]:
        pu.explain_near_tie(int(t), sh, keys, keys, idx, o_idx, kerr)
    o_w = oracle.gate_weights(keys, idx, sh.gate, sh.renormalize, sh.routed_scale)
    np.testing.assert_allclose(w, o_w, rtol=0, atol=1e-5 * max(1.0, sh.routed_scale))
    ref = reference(inputs, idx, o_w)
    err = pu.rel_fro(got, ref)
    assert err <= pu.REL_TOL, f"{err:.2e}"
    for t in range(sh.T):
        if np.linalg.norm(ref[t]) > 0:
            assert pu.rel_fro(got[t], ref[t]) <= 2 * pu.REL_TOL, t
        else:
            assert (got[t] == 0).all(), t
    return layer, got


SMALL = MoEShape(T=5, d=256, E=16, top_k=4, F=96, E_local=16)


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("T", [1, 2, 7, 15, 16, 17, 31, 33, 63, 64])
def test_token_counts(T, mixed):
    check(SMALL.replace(T=T, F_shared=64), mixed)


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("d,F,Fs", [(32, 32, 0), (64, 32, 32), (288, 416, 160), (1056, 1408, 96), (2048, 768, 768),
                                    (7168, 64, 0)])
def test_widths(d, F, Fs, mixed):
    check(SMALL.replace(d=d, F=F, F_shared=Fs), mixed)


@pytest.mark.parametrize("d,F,Fs", [(8, 8, 8), (40, 24, 0), (264, 1000, 40), (2040, 104, 72)])
def test_widths_bf16(d, F, Fs):
    """bf16 weights take any multiple of 8."""
    check(SMALL.replace(d=d, F=F, F_shared=Fs), False)


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("kw", [
    dict(E=2, E_local=2, top_k=1, T=40),                              # up to 40 rows for one expert
    dict(E=1, E_local=1, top_k=1, T=64),                              # 64 rows for one expert
    dict(E=7, E_local=3, e_begin=2, top_k=3, T=30),                   # a slice from the middle, an odd count
    dict(E=384, E_local=1, e_begin=383, top_k=2, T=3),                # most tokens have no local expert
    dict(E=1024, E_local=1024, top_k=16, T=9, F=32),                  # as many experts and choices as there can be
    dict(E=64, E_local=64, top_k=8, T=64, gate=GATE_SIGMOID, n_group=8, topk_group=3, routed_scale=2.5),
    dict(E=40, E_local=20, e_begin=20, top_k=6, T=12, renormalize=0),
    dict(E=40, E_local=40, top_k=6, T=12, renormalize=0, gate=GATE_SIGMOID, F_shared=32),
    dict(E=16, E_local=16, top_k=4, T=33, expert_capacity=3),         # later slots are dropped
    dict(E=4, E_local=4, top_k=2, T=64, expert_capacity=20, F_shared=64),
    dict(E=4, E_local=4, top_k=2, T=64, expert_capacity=1),
])
def test_routing_forms(kw, mixed):
    check(SMALL.replace(**kw), mixed, seed=3)


@pytest.mark.parametrize("mixed", [False, True])
def test_router_bias(mixed):
    check(SMALL.replace(T=21), mixed, zipf_s=1.2)


def test_no_local_expert_at_all():
    """Tokens whose every choice lies elsewhere: zeros, or the shared expert alone."""
    sh = MoEShape(T=4, d=64, E=64, top_k=1, F=32, E_local=1, e_begin=0)
    inputs = make(sh, False, seed=1)
    keys = oracle.bf16_to_f64(inputs["x"]) @ oracle.bf16_to_f64(inputs["w_router"]).T
    e = int(np.setdiff1d(np.arange(64), keys.argmax(1))[0])
    for Fs in (0, 32):
        _, got = check(sh.replace(e_begin=e, F_shared=Fs), False, seed=1)
        assert Fs or (got == 0).all()


@pytest.mark.parametrize("mixed", [False, True])
def test_workload_decode_step(mixed):
    """The decode workload's own shape on fewer experts, and the crossover shape's."""
    k2 = wl.WORKLOADS["k2decode"].shape
    check(k2.replace(E=96, E_local=6, top_k=4, T=32), mixed)
    check(wl.crossover(2).shape.replace(T=64), mixed)


def test_matches_the_layer():
    """bf16 weights: the routing of moe_layer_forward (same keys up to the order of sums) and its result within both
    sides' roundings: each is within REL_TOL of the oracle."""
    inputs = make(SMALL.replace(T=48, F_shared=96, F=256, d=512), False)
    layer = moe.DeviceLayer(inputs)
    a = layer.forward().double().cpu().numpy()
    b = layer.decode().double().cpu().numpy()
    assert pu.rel_fro(b, a) <= 2 * pu.REL_TOL


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("T,kw", [
    (1, dict(E=1, E_local=1, top_k=1)),
    (4, dict(E=2, E_local=2, top_k=1)),                               # tokens that share experts
    (4, dict(E=4, E_local=4, top_k=4, F_shared=96)),                  # every token chooses every expert
    (4, dict(E=8, E_local=8, top_k=8)),                               # 32 slots
    (3, dict(E=16, E_local=16, top_k=11)),                            # 33
    (4, dict(E=16, E_local=16, top_k=16)),                            # 64
    (3, dict(E=65, E_local=30, e_begin=20, top_k=5)),
    (2, dict(E=130, E_local=130, top_k=6, gate=GATE_SIGMOID, routed_scale=2.5)),
    (4, dict(E=256, E_local=256, top_k=8, gate=GATE_SIGMOID, n_group=8, topk_group=3)),
    (4, dict(E=255, E_local=255, top_k=4, n_group=5, topk_group=2)),  # groups that are no runs of lanes
    (1, dict(E=512, E_local=512, top_k=16)),
    (2, dict(E=513, E_local=513, top_k=4)),
    (2, dict(E=300, E_local=3, e_begin=297, top_k=2)),                # most likely nobody's expert
    (4, dict(E=3, E_local=3, top_k=2, expert_capacity=1)),            # dropped slots
    (4, dict(E=4, E_local=2, e_begin=1, top_k=3, expert_capacity=2, F_shared=32)),
    (2, dict(E=16, E_local=16, top_k=4, d=512, F=4096)),              # more workgroups than are on the chip at once
])
def test_few_tokens_routing(T, kw, mixed):
    """Up to a token per wave and a slot per lane the gates are made where they are used; and just past that."""
    check(SMALL.replace(T=T, **kw), mixed)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 3.0e38])
@pytest.mark.parametrize("mixed", [False, True])
def test_a_token_of_no_finite_values_stays_alone(bad, mixed):
    """Wherever such a token is sent, the other tokens' results do not change by a bit."""
    sh = SMALL.replace(T=21, F_shared=64)
    inputs = make(sh, mixed)
    layer = moe.DeviceLayer(inputs)
    layer.quantize()
    good = layer.decode(mx=mixed).clone()
    layer.x[13] = bad
    got = layer.decode(mx=mixed)
    others = torch.arange(sh.T, device="cuda") != 13
    assert torch.equal(got[others], good[others])
    assert not torch.isfinite(got[13]).all()
    idx = routing(layer)[0]
    assert ((idx >= 0) & (idx < sh.E)).all()


@pytest.mark.parametrize("mixed", [False, True])
def test_weight_offsets_past_32_bits(mixed):
    """160 experts of 2048 x 7168: the last ones' weights lie past 2^31 values and, in bf16, past 2^32; a router bias
    sends every token to the last four."""
    T, d, F, E = 3, 7168, 2048, 160
    sh = MoEShape(T=T, d=d, E=E, top_k=4, F=F, E_local=E)
    g = torch.Generator(device="cuda").manual_seed(12)
    x = torch.empty((T, d), device="cuda").normal_(generator=g).to(torch.bfloat16)
    router = (torch.empty((E, d), device="cuda").normal_(generator=g) * d ** -0.5).to(torch.bfloat16)
    bias = torch.zeros(E, device="cuda")
    bias[-4:] = 100.0
    kept = {}
    w = {}
    for name, rows, K in (("w13", 2 * F, d), ("w2", d, F)):
        last = (torch.empty((4 * rows, K), device="cuda").normal_(generator=g) * K ** -0.5).to(torch.bfloat16)
        if mixed:
            q, s = (torch.empty((E * rows, n), dtype=torch.uint8, device="cuda") for n in (K // 2, K // 32))
            q.fill_(0x77), s.fill_(254)                        # what other experts hold would be seen
            moe.moe_mx_quantize(mx.E2M1, last, q[-4 * rows:], s[-4 * rows:])
            moe.moe_mx_dequantize(mx.E2M1, q[-4 * rows:], s[-4 * rows:], last)
            w[name] = (q, s)
        else:
            w[name] = (torch.full((E * rows, K), float("nan"), dtype=torch.bfloat16, device="cuda"), None)
            w[name][0][-4 * rows:] = last
        kept[name] = last.double().cpu().numpy().reshape(4, rows, K)
    out, ws = torch.empty_like(x), moe.alloc_workspace(sh, moe.MOE_WS_DECODE)
    moe.moe_layer_decode(sh, x, router, bias, w["w13"][0], w["w2"][0], None, None, out, ws,
                         (w["w13"][1], w["w2"][1], None, None) if mixed else None)
    xv, L = x.double().cpu().numpy(), x.double().cpu().numpy() @ router.double().cpu().numpy().T + bias.double().cpu().numpy()
    gates = np.exp(L[:, -4:] - L.max(1, keepdims=True))
    gates /= gates.sum(1, keepdims=True)
    ref = sum(gates[:, i:i + 1] * oracle.swiglu_ffn(xv, kept["w13"][i], kept["w2"][i]) for i in range(4))
    assert pu.rel_fro(out.double().cpu().numpy(), ref) <= pu.REL_TOL


@pytest.mark.parametrize("mixed", [False, True])
def test_repeats_bit_for_bit_and_in_a_used_workspace(mixed):
    layer, first = check(SMALL.replace(T=40, F_shared=64), mixed)
    for fill in (0, 255, 0x7f):
        layer.ws_decode.fill_(fill)
        assert np.array_equal(layer.decode(mx=mixed).double().cpu().numpy(), first)


@pytest.mark.parametrize("mixed", [False, True])
def test_replays_in_a_graph(mixed):
    sh = SMALL.replace(T=9, F_shared=64)
    layer = moe.DeviceLayer(make(sh, mixed))
    layer.quantize()
    layer.decode(mx=mixed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.decode(mx=mixed)
    eager = moe.DeviceLayer(make(sh, mixed))
    eager.mx = layer.mx
    eager.x = layer.x
    rng = np.random.default_rng(0)
    for i in range(5):
        layer.x.copy_(moe.to_device_bf16(f32_to_bf16_bits(rng.standard_normal((9, sh.d)).astype(np.float32))))
        graph.replay()
        got = layer.out.clone()
        want = eager.decode(mx=mixed)
        torch.cuda.synchronize()
        assert torch.equal(got, want), i


def test_two_calls_at_once():
    """Two layers on two streams, each with its own workspace, many times over."""
    shapes = [SMALL.replace(T=33, F_shared=64, F=512, d=1024), SMALL.replace(T=1, F=768, d=2048)]
    layers = [moe.DeviceLayer(make(s, False, seed=i)) for i, s in enumerate(shapes)]
    want = [l.decode().clone() for l in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    outs = [[], []]
    for _ in range(20):
        for k, (l, s) in enumerate(zip(layers, streams)):
            with torch.cuda.stream(s):
                l.decode()
                outs[k].append(l.out.clone())
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(o, want[k]) for o in outs[k])
