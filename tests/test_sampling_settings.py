"""What Settings makes of one setting for all rows."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_16450_gb300 import sampling as sp  # noqa: E402


@pytest.mark.parametrize("name,off,on", [("top_p", (1.0, 2.0, math.inf), (0.999, 0.0, -1.0)),
                                         ("min_p", (0.0, -0.0, -1.0, -math.inf), (1e-30, 0.5, 2.0))])
def test_filters_that_are_off(name, off, on):
    for x in off:
        assert sp.Settings(**{name: x}).rows(2, "cpu")[name] is None
    for x in on:
        assert sp.Settings(**{name: x}).rows(2, "cpu")[name].tolist() == [float(torch.tensor(x))] * 2


@pytest.mark.parametrize("name", ["temperature", "top_p", "min_p"])
def test_nan_reaches_the_kernel(name):
    """Which refuses its rows, as those of the same number in a tensor."""
    assert sp.Settings(**{name: math.nan}).rows(2, "cpu")[name].isnan().all()
