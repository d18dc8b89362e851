"""The arithmetic that the paged attention's softmax rests on, compiled for the
host: how a row's reference moves."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_16450_gb300", "csrc")
SOURCE = """
#include "paged_math.h"
using namespace ebd;
// the kernel's loop for a row whose largest score is y: the moves made, and what
// is left of y; probabilities are scaled by 2^-lost
extern "C" int settle(float y, float* ref, int* started, float* left, float* lost) {
  int moves = 0;
  bool s = *started != 0;
  *lost = 0.f;
  for (;; ++moves) {
    const float top = *left = y - *ref;
    if (!(moves < kPagedMoves && paged_far(top, s))) break;
    *lost += paged_move(top, *ref, s);
  }
  *started = s;
  return moves;
}
extern "C" float product_ref(float m, float top) { return paged_product_ref(m, top); }
extern "C" int coarse(float ref) { return paged_coarse(ref); }
extern "C" int most_moves() { return kPagedMoves; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("paged_math")
    (d / "m.cpp").write_text(SOURCE)
    subprocess.run([cxx, "-std=c++17", "-O1", "-ffp-contract=off", "-shared", "-fPIC", "-I", CSRC, str(d / "m.cpp"),
                    "-o", str(d / "m.so")], check=True)
    m = ctypes.CDLL(str(d / "m.so"))
    f = ctypes.POINTER(ctypes.c_float)
    m.product_ref.argtypes, m.product_ref.restype = [ctypes.c_float] * 2, ctypes.c_float
    m.coarse.argtypes = [ctypes.c_float]
    m.settle.argtypes = [ctypes.c_float, f, ctypes.POINTER(ctypes.c_int), f, f]
    return m


class Row:
    """A row's reference, and what it has lost of its first probabilities."""

    def __init__(self, lib, ref=0.0, started=0):
        self.lib, self.ref, self.started = lib, ctypes.c_float(ref), ctypes.c_int(started)

    def settle(self, y):
        left, lost = ctypes.c_float(), ctypes.c_float()
        moves = self.lib.settle(y, *(ctypes.byref(x) for x in (self.ref, self.started, left, lost)))
        return moves, left.value, lost.value


def _scores(rng, n):
    """Floats of every binade from 2^-10 to 2^127, of either sign."""
    x = rng.uniform(1, 2, n) * np.exp2(rng.integers(-10, 128, n))
    return (np.where(rng.random(n) < 0.5, -x, x)).astype(np.float32)


def test_a_reference_reaches_any_score_in_a_few_moves(lib):
    """Scores one after the other, each larger than the row's reference by any
    distance: the moves end by themselves, leave little of the score on either
    side, and what is lost is the reference's move, or everything."""
    rng = np.random.default_rng(0)
    most = 0
    for trial in range(4000):
        ys = _scores(rng, 6)
        ys = np.sort(np.concatenate([ys, np.nextafter(ys, np.float32(np.inf)), ys + np.float32(30.0)]))
        row = Row(lib)
        for y in ys[np.isfinite(ys)].astype(np.float32).tolist():
            was, started = row.ref.value, row.started.value
            moves, left, lost = row.settle(y)
            most = max(most, moves)
            assert moves < lib.most_moves() and row.started.value
            assert -2.0 < left <= 24.0
            if started and moves:
                assert lost == np.inf or (lost == np.ceil(lost) and abs(row.ref.value - was - lost) <= 0.5)
                assert lost < np.inf or y - was >= 2.0 ** 23
    assert most == 2


def test_scores_that_are_infinite_or_nan_end_too(lib):
    for y in (np.inf, -np.inf, np.nan):
        for r in (0.0, 1e9, -3e38, 3e38, np.inf):
            for started in (0, 1):
                assert Row(lib, r, started).settle(float(y))[0] <= lib.most_moves()


def test_products_stay_in_range_of_f16_for_scores_of_any_size(lib):
    """Keys of a row with scores y and value scales 2^d, d in [-40, 0]: against the
    reference the largest product 2^(y - ref + d) is 2^7 (2^8 at most where 32 bits
    do not resolve that), and the largest score's probability is not lost."""
    rng = np.random.default_rng(2)
    f = np.float32
    coarse = 0
    for trial in range(4000):
        x = _scores(rng, 1)[0]
        # scores that differ by log2 units where these resolve, and by units of x's last place
        y = np.concatenate([[x], x - f(60) * rng.random(4).astype(f), x - rng.integers(0, 3, 4).astype(f) * np.spacing(abs(x))])
        d = rng.integers(-40, 1, y.size).astype(f)
        top = (y + d).max()
        large = lib.coarse(float(top))
        coarse += large
        if large:  # the largest score in its place
            top = y.max()
        left = y - f(lib.product_ref(-math.inf, float(top)))
        most = float((left + d).max())
        assert left.max() >= 0 and (most <= 8 if large else abs(most - 7) <= 0.75)
    assert coarse > 1000 and not lib.coarse(-math.inf)
    assert lib.product_ref(-math.inf, -math.inf) == -math.inf and lib.product_ref(5.0, -math.inf) == 5.0
