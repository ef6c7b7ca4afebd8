"""The block-scaled expert MLP on every tile that its rules choose: each case names the tile of its up- and its
down-projection (test_mx_tile_rule.py checks that it gets there), with loads that end in every part of a tile."""
import numpy as np
import pytest
import torch

import mx_util as mx
import test_gpu_operators_together as together
from paper_2607_18631_amd import moe
from paper_2607_18631_amd.workloads import MoEShape

pytestmark = pytest.mark.gpu
U8 = torch.uint8


def spread(first, groups, total):
    """`first`, then groups up to `groups` around the mean of what is left of `total`."""
    n = groups - len(first)
    mean = (total - sum(first)) // n
    return first + [max(0, mean + (i % 3 - 1) * (mean // 3)) for i in range(n)]


FEW = [130, 0, 128, 129, 1, 127]
MANY = spread([0, 1, 63, 64, 65, 127, 128, 129, 192, 193, 255, 256, 257], 32, 1950)
FULL = spread([300, 257, 0, 1, 63, 64, 65, 127, 128, 129, 191, 192, 255, 256, 513], 64, 64 * 72)
# (d, F, rows of each expert, tile of the up-projection, of the down-projection)
CASES = [
    (512, 640, FEW, "128x128", "128x128"),          # K of whole slices
    (544, 608, FEW, "128x128", "128x128"),          # and not
    (1280, 1024, MANY, "128x256", "128x256"),       # K of whole slices of 256
    (1152, 1152, MANY, "128x256", "128x256"),       # of 128
    (1184, 1056, MANY, "128x256", "128x256"),       # and of neither
    (1024, 512, FULL, "256x256", "256x256"),
    (1152, 640, FULL, "256x256", "256x256"),
    (1056, 544, FULL, "256x256", "256x256"),
]
IDS = [f"{d}x{F}-{len(c)}" for d, F, c, *_ in CASES]


def run(sh, fmt, w, x, counts, w13=None, s13=None, w2=None, s2=None):
    n, d = x.shape
    q, s = torch.empty((n, moe.mx_elements_per_row(fmt, d)), dtype=U8, device="cuda"), torch.empty((n, d // 32), dtype=U8, device="cuda")
    moe.moe_mx_quantize(fmt, x, q, s)
    offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    y = torch.full((n, d), -77.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_mx_grouped_ffn(sh, fmt, q, s, offsets, w13, s13, w2, s2, y, moe.alloc_workspace(sh, moe.MOE_WS_MX_FFN))
    return y


@pytest.mark.parametrize("fmt", [mx.E2M1, mx.E4M3], ids=["e2m1", "e4m3"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_every_tile(case, fmt):
    """Against float64 (5e-3 of the norm: two roundings and the activation's rounding borders; an expert of few rows twice
    that), and bit for bit what the expert gives alone, on the smallest tile: a sum's order is not its tile's."""
    d, F, counts = case[:3]
    E, n = len(counts), sum(counts)
    sh = MoEShape(T=n, d=d, E=E, top_k=1, F=F, E_local=E)
    w = together.Experts(sh, 7)
    x = together.normal(d, n, d)
    y = run(sh, fmt, w, x, counts, w.w13, w.w13_scales, w.w2, w.w2_scales)
    rows = mx.rounded(together.f64(x), fmt)
    got, at, num, den = together.f64(y), 0, 0.0, 0.0
    for e, m in enumerate(counts):
        if m == 0:
            continue
        ref = w.mlp(e, rows[at:at + m], lambda a: mx.rounded(a, fmt))
        off, size = np.sum((got[at:at + m] - ref) ** 2), np.sum(ref ** 2)
        assert np.sqrt(off / size) <= 1e-2, (e, m, np.sqrt(off / size))
        num, den = num + off, den + size
        if e < 16:
            one = MoEShape(T=m, d=d, E=1, top_k=1, F=F, E_local=1)
            alone = run(one, fmt, w, x[at:at + m], [m], w.w13[e * 2 * F:(e + 1) * 2 * F], w.w13_scales[e * 2 * F:(e + 1) * 2 * F],
                        w.w2[e * d:(e + 1) * d], w.w2_scales[e * d:(e + 1) * d])
            assert torch.equal(alone, y[at:at + m]), (e, m)
        at += m
    assert np.sqrt(num / den) <= 5e-3, np.sqrt(num / den)
