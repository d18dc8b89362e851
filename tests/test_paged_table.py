"""The host side of the paged K/V cache: which pages hold which sequence."""
import numpy as np
import pytest

from paper_2609_16450_gb300.paged import OutOfPages, PageTable


def _check(t: PageTable):
    """Every page is free or one sequence's, rows are filled from the left."""
    used = t.table[t.table >= 0]
    assert sorted(used.tolist() + t._free) == list(range(t.n_pages))
    for row, n in zip(t.table, t.held):
        assert (row[:n] >= 0).all() and (row[n:] == -1).all()


def test_reserve_grows_and_keeps():
    t = PageTable(8, 2, 5, 16)
    assert t.reserve(0, 17) and t.held[0] == 2
    first = t.table[0, :2].copy()
    assert not t.reserve(0, 32) and not t.reserve(0, 0)
    assert t.reserve(0, 33) and (t.table[0, :2] == first).all() and t.held[0] == 3
    assert t.free == 5
    _check(t)


def test_release_gives_back_the_tail():
    t = PageTable(8, 2, 5, 16)
    t.reserve(0, 80)
    kept = t.table[0, :2].copy()
    assert t.release(0, 20) and t.held[0] == 2 and (t.table[0, :2] == kept).all()
    assert not t.release(0, 32)
    assert t.release(0) and t.free == 8 and not t.release(0)
    _check(t)


def test_out_of_pages_changes_nothing():
    t = PageTable(4, 2, 4, 16)
    t.reserve(0, 40)
    before = t.table.copy()
    with pytest.raises(OutOfPages):
        t.reserve(1, 20)
    assert (t.table == before).all() and t.free == 1
    t.release(0)
    assert t.reserve(1, 64)
    _check(t)


@pytest.mark.parametrize("call", [lambda t: t.reserve(2, 1), lambda t: t.reserve(-1, 1), lambda t: t.release(2),
                                  lambda t: t.reserve(0, 81)])
def test_refusals(call):
    t = PageTable(8, 2, 5, 16)
    with pytest.raises(ValueError):
        call(t)
    _check(t)


@pytest.mark.parametrize("args", [(0, 1, 1, 16), (1, 0, 1, 16), (1, 1, 0, 16), (1, 1, 1, 8), (1, 1, 1, 48), (1, 1, 1, 512)])
def test_sizes_are_checked(args):
    with pytest.raises(ValueError):
        PageTable(*args)


def test_random_traffic():
    rng = np.random.default_rng(0)
    t = PageTable(40, 6, 12, 32)
    for _ in range(500):
        s = int(rng.integers(6))
        try:
            if rng.random() < 0.6:
                t.reserve(s, int(rng.integers(0, 12 * 32 + 1)))
            else:
                t.release(s, int(rng.integers(0, 200)) if rng.random() < 0.5 else 0)
        except OutOfPages:
            assert t.free < 12
        _check(t)
