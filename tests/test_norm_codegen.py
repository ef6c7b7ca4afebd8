"""Code generation of the norm (CPU only): the forward's statistics are float64, the backward's sums float32, and nothing
is spilled."""
import os
import re
import shutil

import pytest

from test_serving_codegen import HIPCC, _device_asm

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    text = _device_asm("norm_mx.hip", str(tmp_path_factory.mktemp("asm") / "norm.s"))
    return {f.split(":", 1)[0]: [l.split(";")[0].strip() for l in f.split("\n")] for f in re.split(r"\n(?=_Z\S+:)", text)
            if re.match(r"_Z\S*k_add_norm\S*:", f)}


def test_nothing_is_spilled(kernels):
    assert len(kernels) >= 21
    for name, lines in kernels.items():
        assert not any(l.startswith("scratch_") for l in lines), name


def test_types_of_the_sums(kernels):
    """Six exchanges of a row's sum over a wave, each of one register in float32 and of two in float64."""
    seen = {False: 0, True: 0}
    for name, lines in kernels.items():
        backward = "k_add_norm_bwd" in name
        wide = [l for l in lines if re.match(r"v_\w+_f64", l)]
        if backward:
            assert not wide, (name, wide[:3])
            assert sum(l.startswith("ds_bpermute") for l in lines) <= 6, name
        else:
            assert any(l.startswith("v_fma_f64") for l in wide) and any(l.startswith("v_mul_f64") for l in wide), name
        seen[backward] += 1
    assert seen[False] >= 7 and seen[True] >= 14
