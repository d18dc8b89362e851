"""The sampler's arithmetic, compiled for the host, at the ends of float's range and as
a compiler that fuses products and sums would have it."""
import ctypes
import shutil
import subprocess

import numpy as np
import pytest

from tests.test_sample_math import CSRC, SOURCE, lib  # noqa: F401

LOWEST = np.finfo(np.float32).min


@pytest.mark.parametrize("hi", [0.0, -1.0, -1e31, -1.02e31, -1.6e31, -1.04e32, -3.4e38])
def test_least_logit_below_the_range(lib, hi):  # noqa: F811
    """Of finite logits, min-p keeps all from there up."""
    for m in (LOWEST, np.nextafter(LOWEST, np.float32(0)), np.float32(-3.3e38)):
        border = float(m) + float(np.float32(hi))
        least = np.float32(lib.least(m, np.float32(hi), 0.0))
        if border <= float(LOWEST):
            assert least == LOWEST
        else:
            assert float(least) >= border > float(np.nextafter(least, np.float32(-np.inf)))


def test_weights_where_products_and_sums_may_be_fused(tmp_path):
    """The product whose rounding is made up for is rounded by itself: weights are bit for
    bit those of a build that fuses nothing (on machines that have fused multiply-adds for a
    compiler to use)."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    libs = []
    for flag in ("-ffp-contract=off", "-ffp-contract=fast"):
        so = tmp_path / (flag[2:] + ".so")
        src = tmp_path / "m.cpp"
        src.write_text(SOURCE)
        subprocess.run([cxx, "-std=c++17", "-O2", flag, "-shared", "-fPIC", "-I", CSRC, str(src), "-o", str(so)], check=True)
        m = ctypes.CDLL(str(so))
        m.weights.argtypes = [ctypes.c_float, ctypes.c_float, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
        libs.append(m)
    rng = np.random.default_rng(6)
    for T in (1.0, 0.3, 1.7):
        l = np.float32(-rng.uniform(0, 27.7, 20000) * T)
        w = [np.empty(len(l), np.uint64) for _ in libs]
        for m, out in zip(libs, w):
            m.weights(np.float32(0), np.float32(T), l.ctypes.data, len(l), out.ctypes.data)
        assert np.array_equal(*w)
