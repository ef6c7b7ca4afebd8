"""The cases on which the GPU tests of the block-scaled expert MLP run reach every kernel of its product: the rules of
mx_tile_rule.hpp, compiled for the host, evaluated for the 256 CUs of an MI355X.  A change of a rule that takes a kernel
out of the tests fails here."""
import ctypes
import os
import shutil
import subprocess

import pytest

import test_gpu_mx_tiles as tiles

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2607_18631_amd", "csrc")
CUS = 256
TILES = ["128x128", "128x256", "256x256"]
RAGGED, WHOLE128, WHOLE256 = range(3)

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rule") / "mx_rule.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC,
                    os.path.join(HERE, "mx_tile_rule.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    l = ctypes.c_long
    lib.tile.argtypes = [l, l, l, l]
    lib.slices.argtypes = [ctypes.c_int, ctypes.c_int, l]
    return lib


def products(rule, d, F, counts):
    """(tile, K) of the up- and the down-projection."""
    rows, groups = sum(counts), len(counts)
    return [(TILES[rule.tile(CUS, rows, groups, n)], K) for n, K in ((2 * F, d), (d, F))]


@pytest.mark.parametrize("case", tiles.CASES, ids=tiles.IDS)
def test_cases_reach_their_tiles(rule, case):
    d, F, counts, up, down = case
    assert [t for t, _ in products(rule, d, F, counts)] == [up, down]


def test_cases_reach_every_kernel(rule):
    seen = set()
    for d, F, counts, *_ in tiles.CASES:
        for product, (tile, K) in zip(("up", "down"), products(rule, d, F, counts)):
            for e2m1 in (0, 1):
                seen.add((e2m1, product, tile, rule.slices(e2m1, int(tile.split("x")[1]), K)))
    want = {(e2m1, product, tile, s) for e2m1 in (0, 1) for product in ("up", "down") for tile in TILES
            for s in (RAGGED, WHOLE128, WHOLE256) if s < WHOLE256 or (e2m1 and tile != "128x128")}
    assert len(want) == 28
    assert seen == want


@pytest.mark.parametrize("tile", TILES)
def test_cases_end_in_every_part_of_a_tile(tile):
    """A group's last rows fill 1 to 64, 65 to 128, more, or all of a tile (the large ones then run on a part of theirs),
    with and without whole tiles before them, on both sides of each border; and a group has none."""
    bm = int(tile.split("x")[0])
    for d, F, counts, up, down in tiles.CASES:
        if up != tile:
            continue
        last = {(c - 1) % bm + 1 for c in counts if c}
        assert {1, bm - 1, bm} <= last and 0 in counts and max(counts) > bm
        if tile != "128x128":
            assert {1, 63, 64, 65, 127, 128} <= last
        if bm == 256:
            assert {129, 255, 256} <= last


def test_rule_at_its_borders(rule):
    # as many 128 x 128 tiles as compute units, and one group more
    assert rule.tile(CUS, 16 * 64, 16, 2048) == 0 and rule.tile(CUS, 17 * 64, 17, 2048) == 1
    # 64 rows a group, and 65
    assert rule.tile(CUS, 64 * 64, 64, 1024) == 1 and rule.tile(CUS, 64 * 65, 64, 1024) == 2
    assert [rule.slices(1, 256, K) for K in (256, 384, 512, 576, 640, 768)] == [0, 0, 2, 0, 1, 2]
    assert [rule.slices(0, 256, K) for K in (384, 512, 640, 672)] == [0, 1, 1, 0]
    assert [rule.slices(1, 128, K) for K in (384, 512, 640, 672)] == [0, 1, 1, 0]
