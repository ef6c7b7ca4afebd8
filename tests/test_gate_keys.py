"""The integer images of the gate's keys (order_key.hpp, compiled for the host): the keys' order, and never the 0 that
marks an expert that cannot be chosen, whatever bits a key has."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2607_18631_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")


@pytest.fixture(scope="module")
def images(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("keys") / "keys.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC,
                    os.path.join(HERE, "order_key.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.images.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_long]

    def call(bits):
        bits = np.ascontiguousarray(bits, np.uint32)
        image, back = np.empty_like(bits), np.empty_like(bits)
        lib.images(bits.ctypes.data, image.ctypes.data, back.ctypes.data, bits.size)
        return image, back
    return call


# every sign and exponent with the mantissas at both ends and in between
MANTISSAS = np.array([0, 1, 2, 0x3fffff, 0x400000, 0x400001, 0x7ffffe, 0x7fffff], np.uint32)
ALL = (np.arange(512, dtype=np.uint32)[:, None] << 23 | MANTISSAS).ravel()


def test_no_key_is_the_mark_of_an_expert_that_cannot_be_chosen(images):
    assert 0xffffffff in ALL
    assert (images(ALL)[0] > 0).all()


def test_order_and_inverse(images):
    v = ALL.view(np.float32)
    bits = ALL[~np.isnan(v)]
    bits = bits[np.argsort(bits.view(np.float32), kind="stable")]
    image, back = images(bits)
    v = bits.view(np.float32)
    assert ((np.diff(v.astype(np.float64)) > 0) == (np.diff(image.astype(np.int64)) > 0))[np.isfinite(v[1:]) & np.isfinite(v[:-1])].all()
    assert (np.diff(image.astype(np.int64)) >= 0).all()
    np.testing.assert_array_equal(back.view(np.float32), v)          # (-0 comes back as +0)
    for inf, inside in ((0x7f800000, 0x7f7fffff), (0xff800000, 0xff7fffff)):
        a, b = images([inf])[0][0], images([inside])[0][0]
        assert a > b if inf < 0x80000000 else a < b


def test_a_nan_comes_back_as_a_nan(images):
    nan = ALL[np.isnan(ALL.view(np.float32))]
    assert np.isnan(images(nan)[1].view(np.float32)).all()
