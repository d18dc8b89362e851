"""The plans that the device's are compared with, against the host's page table."""
import random

from paper_2609_16450_gb300.paged import PageTable
from tests.plan_ref import Plan


def test_plans_are_the_page_tables():
    rng = random.Random(0)
    ref, t = Plan(40, 6, 9, 16), PageTable(40, 6, 9, 16)
    ref.free = list(t._free)
    for _ in range(200):
        add = [rng.choice((0, 1, rng.randint(0, 40), -rng.randint(1, 80))) for _ in range(6)]
        old = list(ref.len)
        rows = ref.step(add, 10 ** 6)
        if rows is None:
            assert ref.len == old
            continue
        for b in reversed(range(6)):
            if ref.len[b] < old[b]:
                t.release(b, ref.len[b])
        for b in range(6):
            t.reserve(b, ref.len[b])
        assert t.table.tolist() == ref.table and t._free == ref.free
        cu, pos, slot = rows
        for b in range(6):
            assert pos[cu[b]: cu[b + 1]] == list(range(old[b], old[b] + max(add[b], 0)))
            assert all(s // 16 == ref.table[b][p // 16] for p, s in zip(pos[cu[b]: cu[b + 1]], slot[cu[b]: cu[b + 1]]))


def test_a_plan_that_cannot_be_met_changes_nothing():
    ref = Plan(4, 2, 3, 16)
    ref.step([20, 17])
    state = ([list(x) for x in ref.table], list(ref.free), list(ref.len))
    assert ref.step([1, 16 * 2]) is None and ref.step([49 - 20, 0]) is None and ref.step([1, 1], 1) is None
    assert state == (ref.table, ref.free, ref.len)
