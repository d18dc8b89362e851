"""The plain e4m3 quantiser that the GPU tests compare with: pinned by the
format's own values, without a GPU."""
import numpy as np
import pytest

from tests import paged_ref as pr


def test_codes_are_fixed_points():
    val = pr.e4m3_values()
    for c in range(256):
        if c & 0x7F == 0x7F:
            assert np.isnan(val[c])
            continue
        row = np.array([val[c], 448.0])  # 448 fixes the scale at 1
        code, e = pr.quantise(row)
        assert e == 127 and (code[0] == c or (c == 128 and code[0] == 128))


def test_rounding_is_to_the_nearest_code_with_ties_to_even():
    val = pr.e4m3_values()
    pos = val[:0x7F]
    rng = np.random.default_rng(3)
    x = np.concatenate([rng.uniform(0, 448, 2000), (pos[1:] + pos[:-1]) / 2])
    for i in range(0, len(x), 50):
        chunk = x[i: i + 50]
        code, e = pr.quantise(np.concatenate([chunk, [448.0]]))
        assert e == 127
        for a, c in zip(chunk, code):
            d = np.abs(pos - a)
            best = np.flatnonzero(d == d.min())
            assert c in best and (len(best) == 1 or c % 2 == 0)


@pytest.mark.parametrize("amax,k", [(448.0, 0), (448.0 * (1 + 2.0 ** -7), 1), (1.75, -8), (1.7578125, -7), (1.0, -8),
                                    (0.0, -127), (2.0 ** -133, -127), (3.3895e38, 120), (2.0 ** -118, -126)])
def test_scale_is_the_least_power_of_two(amax, k):
    code, e = pr.quantise(np.array([amax, -amax / 2]))
    assert int(e) - 127 == k
    assert amax <= 448 * 2.0 ** k and (k == -127 or amax > 448 * 2.0 ** (k - 1))


def test_values_that_are_not_finite():
    code, e = pr.quantise(np.array([[np.inf, 1.0], [0.5, np.nan], [-np.inf, 0.0], [2.0, 1.0]]))
    assert (code[:3] == 0x7F).all() and list(e[:3]) == [255] * 3 and e[3] == 127 - 7
    back = pr.dequantise(code, e)
    assert np.isnan(back[:3]).all() and list(back[3]) == [2.0, 1.0]
