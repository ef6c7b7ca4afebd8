"""Routers whose keys are no ordinary numbers: every choice stays an expert of its own, and nothing but the tokens
concerned changes."""
import numpy as np
import pytest
import torch

import test_gpu_decode as td
from paper_2607_18631_amd import moe
from paper_2607_18631_amd.workloads import MoEShape

pytestmark = pytest.mark.gpu
SMALL = MoEShape(T=5, d=256, E=16, top_k=4, F=96, E_local=16)


def check_choices(idx, sh):
    assert ((idx >= 0) & (idx < sh.E)).all()
    assert all(len(set(row)) == sh.top_k for row in idx.tolist())


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("T,kw", [
    (1, {}), (4, {}), (4, dict(expert_capacity=64)), (4, dict(E=8, E_local=8, top_k=8, expert_capacity=5)),
    (3, dict(E=300, E_local=300)), (4, dict(E=16, E_local=16, n_group=4, topk_group=2)),
    (21, {}), (64, dict(expert_capacity=3, F_shared=64)), (9, dict(E=1024, E_local=1024, top_k=16, F=32)),
])
def test_a_bias_of_memory_filled_with_ones(T, kw, mixed):
    """A NaN of all ones is the key of every expert, or of all but two: each token still chooses top_k experts, once each
    (an expert's rows then fit where they are kept), and the call after it finds nothing changed."""
    sh = SMALL.replace(T=T, **kw)
    layer = moe.DeviceLayer(td.make(sh, mixed, seed=2))
    layer.quantize()
    layer.bias = torch.zeros(sh.E, device="cuda")
    good, idx = layer.decode(mx=mixed).clone(), td.routing(layer)[0]
    for few in (0, 2):
        layer.bias.view(torch.int32).fill_(-1)
        if few:
            layer.bias[torch.tensor([1, sh.E - 2])] = 0.0
        layer.decode(mx=mixed)
        check_choices(td.routing(layer)[0], sh)
    layer.bias.zero_()
    again = layer.decode(mx=mixed)
    assert torch.equal(again, good) and np.array_equal(td.routing(layer)[0], idx)


@pytest.mark.parametrize("T", [3, 200])
def test_a_bias_of_memory_filled_with_ones_in_the_layer(T):
    sh = SMALL.replace(T=T, F_shared=64)
    layer = moe.DeviceLayer(td.make(sh, False, seed=2))
    layer.bias = torch.zeros(sh.E, device="cuda")
    good = layer.forward().clone()
    layer.bias.view(torch.int32).fill_(-1)
    layer.forward()
    check_choices(layer.region(moe.MOE_REGION_TOPK_IDX, torch.int32, (sh.T, sh.top_k)).cpu().numpy(), sh)
    layer.bias.zero_()
    assert torch.equal(layer.forward(), good)


@pytest.mark.parametrize("d", [8, 72, 256, 320, 1000, 2048, 4104])
def test_infinite_router_weights(d):
    """One infinite weight of an expert, at places all over K: its keys are infinities of the token's sign there, so tokens
    with a negative value never choose it, those with a positive one choose it first, and no other key changes.  (A part of
    K that also reads its neighbour's weights, times zeros, would make every key a NaN.)"""
    T, E, k = 21, 32, 4
    sh = SMALL.replace(T=T, d=d, E=E, E_local=E, top_k=k, F=32)
    layer = moe.DeviceLayer(td.make(sh, False, seed=d))
    layer.x[:, 0] = torch.where(torch.arange(T, device="cuda") % 2 == 0, 1.0, -1.0)
    for i, at in enumerate(sorted({0, 7, d // 3, d // 2 - 1, d // 2, d - 8, d - 1} | set(range(40, d, 152)))):
        at, e = min(at, d - 1), (5 * i + 3) % E
        layer.x[:, at] = layer.x[:, 0]
        logits = (layer.x.double() @ layer.w_router.double().t()).cpu().numpy()
        was = layer.w_router[e, at].clone()
        layer.w_router[e, at] = float("inf")
        layer.decode()
        idx, w = td.routing(layer)
        layer.forward()
        as_layer = layer.region(moe.MOE_REGION_TOPK_IDX, torch.int32, (T, k)).cpu().numpy()
        layer.w_router[e, at] = was
        for t in range(T):
            want = logits[t].copy()
            want[e] = -np.inf if t % 2 else np.inf
            order = np.argsort(-want, kind="stable")
            if t % 2:
                assert e not in idx[t], (at, t)
                assert np.isfinite(w[t]).all()
            else:
                assert idx[t, 0] == e, (at, t)
            # the choices but for keys nearer than the sums' error
            near = np.abs(want[order[k - 1]] - want[order[k]]) <= 2.0 ** -18 * np.abs(logits[t]).max()
            assert near or set(idx[t]) == set(as_layer[t]) == set(order[:k].tolist()), (at, t)
