"""DeviceLayer's 4-bit weights between calls: without a GPU (the conversion replaced), and in a captured graph."""
import numpy as np
import pytest
import torch

from paper_2607_18631_amd import moe
from paper_2607_18631_amd.workloads import MoEShape, f32_to_bf16_bits

SH = MoEShape(T=3, d=256, E=8, top_k=2, F=96, E_local=8, F_shared=64)
NAMES = ("w13", "w2", "ws13", "ws2")


def bare_layer():
    layer = moe.DeviceLayer.__new__(moe.DeviceLayer)
    layer.shape, layer.device = SH, "cpu"
    for name, shape in zip(NAMES, ((8, 192, 256), (8, 256, 96), (128, 256), (256, 64))):
        setattr(layer, name, torch.zeros(shape, dtype=torch.bfloat16))
    return layer


def test_quantize_again_writes_the_same_buffers(monkeypatch):
    monkeypatch.setattr(moe, "moe_mx_quantize", lambda fmt, x, q, s: (q.fill_(1), s.fill_(2)))
    layer = bare_layer()
    first = {n: [t.data_ptr() for t in pair] for n, pair in layer.quantize().items()}
    assert set(first) == set(NAMES)
    assert [tuple(t.shape) for t in layer.mx["w13"]] == [(8 * 192, 128), (8 * 192, 8)]
    assert {n: [t.data_ptr() for t in pair] for n, pair in layer.quantize().items()} == first


def test_a_refused_conversion_leaves_no_half_made_weights(monkeypatch):
    def refuse(fmt, x, q, s):
        if x.shape[1] == 96:
            raise moe.MoEError(moe.MOE_ERR_UNSUPPORTED, "refused")
    monkeypatch.setattr(moe, "moe_mx_quantize", refuse)
    layer = bare_layer()
    with pytest.raises(moe.MoEError, match="refused"):
        layer.quantize()
    assert getattr(layer, "mx", None) is None


@pytest.mark.gpu
def test_a_captured_layer_reads_weights_that_were_converted_again():
    import test_gpu_decode as td
    inputs = td.make(SH, True)
    layer = moe.DeviceLayer(inputs)
    layer.quantize()
    layer.decode(mx=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.decode(mx=True)
    rng = np.random.default_rng(5)
    for _ in range(3):
        for name in NAMES:
            w = getattr(layer, name)
            w.copy_(moe.to_device_bf16(f32_to_bf16_bits((rng.standard_normal(w.shape) * w.shape[-1] ** -0.5).astype(np.float32))))
        layer.quantize()
        graph.replay()
        got = layer.out.clone()
        fresh = moe.DeviceLayer(inputs)
        for name in NAMES:
            setattr(fresh, name, getattr(layer, name))
        fresh.quantize()
        want = fresh.decode(mx=True)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and want.abs().max() > 0
