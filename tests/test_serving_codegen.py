"""Code generation of the block-scaled grouped product and the few-token layer (CPU only): nothing is spilled, the
direct-to-LDS copies keep their wait state behind M0, a stage's copies stand between matrix instructions, and the
few-token layer never waits for all its loads inside its weight loop."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_18631_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")


def _device_asm(src, out):
    from paper_2607_18631_amd import build
    subprocess.run([HIPCC, *build.FLAGS, "-I", CSRC, "-x", "hip", "--cuda-device-only", "-S", os.path.join(CSRC, src), "-o", out],
                   check=True, capture_output=True, text=True)
    with open(out) as f:
        return f.read()


def _mfma_loops(lines):
    """(first, last) lines of the innermost loops (a branch back to a label) with matrix instructions in them."""
    label = {m.group(1): i for i, l in enumerate(lines) if (m := re.match(r"(\.LBB\d+_\d+):", l))}
    back = [re.search(r"s_(?:cbranch_\w+|branch)\s+(\.LBB\d+_\d+)", l) for l in lines]
    loops = [(label[m.group(1)], i) for i, m in enumerate(back) if m and label.get(m.group(1), i) < i]
    loops = [(a, b) for a, b in loops if any(l.startswith("v_mfma") for l in lines[a:b])]
    return [(a, b) for a, b in loops if not any((c, d) != (a, b) and a <= c and d <= b for c, d in loops)]


SOURCES = ["mx_gemm.hip", "decode.hip"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    d = tmp_path_factory.mktemp("asm")
    with ThreadPoolExecutor(len(SOURCES)) as ex:
        texts = list(ex.map(lambda s: _device_asm(s, str(d / (s + ".s"))), SOURCES))
    out = {}
    for src, text in zip(SOURCES, texts):
        fs = re.split(r"\n(?=_Z\S+:)", text)
        out[src] = {f.split(":", 1)[0]: [l.split(";")[0].strip() for l in f.split("\n")] for f in fs if "v_mfma" in f}
    return out


@pytest.mark.parametrize("src,least", [("mx_gemm.hip", 16), ("decode.hip", 9)])
def test_nothing_is_spilled(kernels, src, least):
    assert len(kernels[src]) >= least, list(kernels[src])
    for name, lines in kernels[src].items():
        assert not any(l.startswith("scratch_") for l in lines), name


@pytest.mark.parametrize("src", SOURCES)
def test_wait_state_behind_m0(kernels, src):
    copies = 0
    for name, lines in kernels[src].items():
        ins = [l for l in lines if l and not l.startswith((".", "_"))]
        for i, l in enumerate(ins):
            if l.startswith("global_load_lds"):
                copies += 1
                assert ins[i - 1].startswith("s_nop") and ins[i - 2].startswith("s_mov_b32 m0"), (name, ins[i - 2:i + 1])
    assert copies >= 20


def test_copies_stand_between_products(kernels):
    """In the K loops of the large tiles no more than four copies follow each other without a product."""
    loops = 0
    for name, lines in kernels["mx_gemm.hip"].items():
        for a, b in _mfma_loops(lines):
            body = [l for l in lines[a:b + 1] if l.startswith(("v_mfma", "global_load_lds"))]
            if sum(l.startswith("v_mfma") for l in body) < 16 or not any(l.startswith("global") for l in body):
                continue
            loops += 1
            run = 0
            for l in body + body:
                run = 0 if l.startswith("v_mfma") else run + 1
                assert run <= 4, name
    assert loops >= 4


def test_weight_loop_keeps_loads_in_flight(kernels):
    """Waits inside the loops over the weights leave loads outstanding, but for the one beside new rows in LDS."""
    loops = 0
    for name, lines in kernels["decode.hip"].items():
        if "k_decode_up" not in name and "k_decode_down" not in name:
            continue
        for a, b in _mfma_loops(lines):
            body = lines[a:b + 1]
            if not any(l.startswith("buffer_load") for l in body):
                continue
            loops += 1
            waits = [re.search(r"vmcnt\((\d+)\)", l) for l in body if l.startswith("s_waitcnt")]
            counts = [int(m.group(1)) for m in waits if m]
            assert counts and max(counts) >= 4, (name, counts)
    assert loops >= 8
