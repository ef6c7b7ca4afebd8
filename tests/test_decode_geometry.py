"""The few-token layer's geometry, compiled for the host: what a launch is given holds what its workgroups put there, for
every admitted shape, and the GPU cases reach every kernel and geometry."""
import ctypes
import itertools
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_decode_geometry as cases
from paper_2607_18631_amd import moe
from paper_2607_18631_amd.workloads import MoEShape

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2607_18631_amd", "csrc")
RED_BYTES = 4 * 2 * 64 * 16

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rule") / "geometry.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC,
                    os.path.join(HERE, "decode_geometry.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


def launches(lib, sh, mx):
    """The up- and the down-projection's (ns, K, K of the shared expert, features, geometry)."""
    for ns, features, K, features_s, K_s in ((2, sh.F, sh.d, sh.F_shared, sh.d),
                                             (1, sh.d, sh.F, sh.d if sh.F_shared else 0, sh.F_shared)):
        out = (ctypes.c_int * 7)()
        lib.geometry(sh.T, sh.E, sh.E_local, sh.top_k, features, K, features_s, K_s, ns, mx, out)
        yield ns, K, K_s, features, dict(zip(("tiles", "shared_tiles", "shared", "split", "shared_split", "room", "lds"), out))


def rounds(mx, K, split, room, m):
    """(all rounds of K, those in LDS at once, bytes that m rows take) as the kernel reckons."""
    unit = 256 if mx else 128
    n = -(-(-(-K // unit)) // split)
    per_round = split * unit
    held = max(1, min(n, (room // m - 16) // (2 * per_round)))
    return n, held, m * (2 * min(held * per_round, K) + 16)


def check(lib, sh, mx):
    for ns, K, K_s, features, g in launches(lib, sh, mx):
        assert g["split"] in (1, 2, 4) and g["shared_split"] in (1, 2, 4)
        assert RED_BYTES <= g["lds"] <= lib.most_lds(), (sh, mx, ns, g)
        products = [(K, g["split"])] + ([(K_s, g["shared_split"])] if sh.F_shared else [])
        for k, split in products:
            scales = ns * (64 // split) * (k // 32) if mx else 0
            for m in range(1, min(sh.T, 16) + 1):
                assert scales + rounds(mx, k, split, g["room"], m)[2] <= g["lds"], (sh, mx, ns, m, g)
        assert g["tiles"] * (64 // g["split"]) >= features
        # workgroups of 256 threads in one launch
        slots = sh.T * sh.top_k
        entries = min(sh.E_local, slots) + (slots // 16 if sh.T > 16 else 0)
        assert g["shared"] + entries * g["tiles"] < 1 << 24, (sh, g)


def test_admitted_shapes_fit(lib):
    rng = random.Random(1)
    log = lambda top, step: max(step, int(2 ** rng.uniform(3, top)) // step * step)
    n = 0
    for mx in (False, True):
        edge = itertools.product((1, 2, 15, 16, 17, 64), (32, 16384) if mx else (8, 1048568), (32, 32768) if mx else (8, 1048568),
                                 (0, 32768 if mx else 1048568), ((1, 1, 1), (8, 8, 2), (1024, 1024, 16), (1024, 1, 1)))
        shapes = [MoEShape(T=T, d=d, E=E, top_k=k, F=F, E_local=El, F_shared=Fs) for T, d, F, Fs, (E, El, k) in edge]
        for _ in range(4000):
            step = 32 if mx else 8
            E = int(2 ** rng.uniform(0, 10))
            shapes.append(MoEShape(T=rng.randint(1, 64), d=log(14 if mx else 20, step), E=E, E_local=rng.randint(1, E),
                                   top_k=rng.randint(1, min(16, E)), F=log(15 if mx else 20, step),
                                   F_shared=rng.choice((0, log(15 if mx else 20, step)))))
        for sh in shapes:
            try:
                moe.workspace_size(sh, moe.MOE_WS_DECODE)
            except moe.MoEError:
                continue
            check(lib, sh, mx)
            n += 1
    assert n > 8000


def test_cases_reach_every_kernel_and_geometry(lib):
    seen, in_rounds, at_once = set(), set(), set()
    for kw in cases.CASES:
        sh = cases.BASE.replace(**kw)
        for mx in (False, True):
            for ns, K, K_s, features, g in launches(lib, sh, mx):
                unit = 256 if mx else 128
                whole = K % unit == 0 and (ns == 2 or sh.F_shared % unit == 0)
                seen.add((ns, mx, whole, g["split"]))
                for name, k, split in (("experts", K, g["split"]),) + ((("shared", K_s, g["shared_split"]),) if sh.F_shared else ()):
                    # as many rows as surely happen: all experts' blocks of 64 tokens that choose one of two; one row
                    m = 16 if name == "shared" or (sh.T == 64 and sh.E == 2) else 1
                    n, held, _ = rounds(mx, k, split, g["room"], m)
                    (in_rounds if held < n else at_once).add((ns, mx, name))
    assert seen == set(itertools.product((1, 2), (False, True), (False, True), (1, 2, 4)))
    assert in_rounds == at_once == set(itertools.product((1, 2), (False, True), ("experts", "shared")))
