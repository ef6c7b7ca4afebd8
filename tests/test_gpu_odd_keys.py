"""Routers whose keys are no ordinary numbers: every choice stays an expert of its own, and nothing but the tokens
concerned changes."""
import numpy as np
import pytest
import torch

import parity_util as pu
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
