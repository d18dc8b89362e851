"""The sampler's arithmetic, compiled for the host, at the ends of float's range."""
import numpy as np
import pytest

from tests.test_sample_math import lib  # noqa: F401

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
