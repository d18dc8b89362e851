"""The sampler's arithmetic, compiled for the host: weights against exact ones, the
parts of sums that shares and random numbers take, the least logit that min-p keeps."""
import ctypes
import os
import shutil
import subprocess
from decimal import Decimal, getcontext
from fractions import Fraction

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_16450_gb300", "csrc")
SOURCE = """
#include "sample_math.h"
using namespace ebd;
static SampleEntry* table() {
  static SampleEntry t[kSampleTable];
  for (int j = 0; j < kSampleTable; ++j) t[j] = sample_entry(j);
  return t;
}
extern "C" void weights(float m, float T, const float* l, int n, uint64_t* w) {
  const SampleScale c = sample_scale(sample_temperature(T));
  const SampleEntry* t = table();
  for (int i = 0; i < n; ++i) w[i] = sample_weight(m, l[i], c, t);
}
extern "C" uint64_t part(float x, uint64_t total, int up) { return sample_part(x, total, up != 0); }
extern "C" uint64_t share(float p, uint64_t total) { return sample_share(p, total); }
extern "C" float least(float m, float hi, float lo) { return sample_floor(m, hi, lo); }
extern "C" uint32_t key(float x) { return order_key(x); }
extern "C" float value(uint32_t k) { return order_value(k); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("sample_math")
    (d / "m.cpp").write_text(SOURCE)
    subprocess.run([cxx, "-std=c++17", "-O1", "-ffp-contract=off", "-shared", "-fPIC", "-I", CSRC, str(d / "m.cpp"),
                    "-o", str(d / "m.so")], check=True)
    m = ctypes.CDLL(str(d / "m.so"))
    f, u64 = ctypes.c_float, ctypes.c_uint64
    m.weights.argtypes = [f, f, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
    m.part.argtypes, m.part.restype = [f, u64, ctypes.c_int], u64
    m.share.argtypes, m.share.restype = [f, u64], u64
    m.least.argtypes, m.least.restype = [f, f, f], f
    m.key.argtypes, m.key.restype = [f], ctypes.c_uint32
    m.value.argtypes, m.value.restype = [ctypes.c_uint32], f
    return m


def _weights(lib, m, T, l):
    l = np.ascontiguousarray(l, np.float32)
    w = np.empty(len(l), np.uint64)
    lib.weights(np.float32(m), np.float32(T), l.ctypes.data, len(l), w.ctypes.data)
    return w


@pytest.mark.parametrize("T", [1.0, 0.3, 1.5, 0.011, 33.0, 1e-30, 1e30, 1e-35, 3e38])
@pytest.mark.parametrize("center", [0.0, 9.0, -400.0, 1e-4, 1e30])
def test_weights(lib, T, center):
    """Off by 2^-30 of themselves, half a unit of 2^-43, and half a step of the float that
    is rounded to units, 2^-21 at most and so 2^-46 (in 64 bits numpy's own exponent is off
    by 2^-52 of x, 28 at most, and its exponential by 2^-52)."""
    rng = np.random.default_rng(1)
    t = min(max(float(np.float32(T)), float(np.float32(1e-30))), float(np.float32(1e30)))
    m = np.float32(center + 3 * t) if center + 3 * t > center else np.float32(center)
    l = np.float32(float(m) - np.concatenate([rng.uniform(0, 29, 4000), rng.uniform(0, 1e-3, 500), [0, 27.7, 27.8, 60]]) * t)
    l = np.minimum(l, m)
    w = _weights(lib, m, T, l).astype(np.float64) * 2.0 ** -43
    x = (l.astype(np.float64) - float(m)) / t
    want = np.where(x < -40 * np.log(2), 0, np.exp(np.maximum(x, -1000.0)))
    err = np.abs(w - want)
    dead = np.abs(x / np.log(2) + 40) < 1e-4  # may be on either side of zero
    assert (err[~dead] <= want[~dead] * (2.0 ** -30 + 2.0 ** -46) + 2.0 ** -44 + 2.0 ** -46).all(), err.max()
    assert (w[dead] <= 2.0 ** -39.9).all()
    assert _weights(lib, m, T, [m])[0] == 2 ** 43
    assert (_weights(lib, m, T, [-np.inf]) == 0).all()


def test_weights_fall_with_the_logit(lib):
    """Equal logits weigh the same, and a lower one no more than 2^-30 above."""
    rng = np.random.default_rng(2)
    l = np.sort(rng.standard_normal(200000).astype(np.float32) * 4)
    w = _weights(lib, l[-1], 0.7, l).astype(np.int64)
    assert (w[:-1] - w[1:] <= w[1:] * 2.0 ** -29 + 1).all()


def test_parts_of_sums(lib):
    rng = np.random.default_rng(3)
    xs = [0.0, 1 - 2.0 ** -24, 0.5, 2.0 ** -149, 2.0 ** -126, 0.1] + list(rng.uniform(0, 1, 200)) + list(
        np.exp(rng.uniform(-100, 0, 200)))
    for x in xs:
        x = float(np.float32(x))
        if x >= 1:
            continue
        for total in (1, 2, 2 ** 44, 2 ** 64 - 1, int(rng.integers(1, 2 ** 62)), int(rng.integers(1, 2 ** 30))):
            exact = Fraction(x) * total
            low = exact.numerator // exact.denominator
            assert lib.part(x, total, 0) == low
            assert lib.part(x, total, 1) == low + (exact != low)
            assert lib.share(x, total) == max(1, low + (exact != low))
    assert lib.share(-1.0, 100) == 1


def test_least_logit_of_min_p(lib):
    rng = np.random.default_rng(4)
    getcontext().prec = 60
    for _ in range(20000):
        m = np.float32(rng.standard_normal() * np.exp(3 * rng.standard_normal()))
        x = -np.exp(3 * rng.standard_normal())
        hi = np.float32(x)
        lo = np.float32(x - float(hi))
        f = np.float32(lib.least(m, hi, lo))
        border = Decimal(float(m)) + Decimal(float(hi)) + Decimal(float(lo))
        assert Decimal(float(f)) >= border > Decimal(float(np.nextafter(f, np.float32(-np.inf))))


def test_order(lib):
    x = np.array([-np.inf, -3e38, -1, -1e-45, 0, 1e-45, 1e-38, 2, 3e38, np.inf], np.float32)
    k = [lib.key(v) for v in x]
    assert k == sorted(k) and len(set(k)) == len(k)
    assert [lib.value(v) for v in k] == [float(v) for v in x]
