"""Code generation of the few-token layer's weight loops (CPU only): a wait for all loads stands beside the copies of new
token rows and nowhere else; every other wait leaves the loads of all units but one on their way."""
import os
import re

import pytest

from test_serving_codegen import HIPCC, _device_asm, _mfma_loops

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")


def weight_loops(text):
    """(kernel, 4-bit weights or not, lines) of the loops with matrix instructions and weight loads."""
    for f in re.split(r"\n(?=_Z\S+:)", text):
        m = re.match(r"_Z\S*k_decode_(?:up|down)ILb([01])\S*:", f)
        if not m:
            continue
        lines = [l.split(";")[0].strip() for l in f.split("\n")]
        for a, b in _mfma_loops(lines):
            body = lines[a:b + 1]
            if any(l.startswith("buffer_load") for l in body):
                yield m.group(0), m.group(1) == "1", body


def test_waits_in_the_weight_loops(tmp_path):
    seen = set()
    for name, mx, body in weight_loops(_device_asm("decode.hip", str(tmp_path / "decode.s"))):
        stages = 4 if mx else 3
        loads = sum(l.startswith("buffer_load") for l in body)
        copies = sum(l.startswith("global_load_lds") for l in body)
        assert loads and loads % stages == 0, (name, loads)
        counts = [int(m.group(1)) for l in body if l.startswith("s_waitcnt") and (m := re.search(r"vmcnt\((\d+)\)", l))]
        assert counts.count(0) == copies, (name, copies, counts)
        rest = [c for c in counts if c]
        assert len(rest) >= stages and min(rest) >= loads - loads // stages, (name, loads, counts)
        seen.add(name)
    # up with the gates made outside or inside for four numbers of experts, and down: each in two formats, K whole or not
    assert len(seen) == 2 * 2 * (5 + 1)
