"""ebd_paged_plan against plans made one page at a time."""
import random

import pytest

from tests.plan_ref import Plan

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

I32 = dict(dtype=torch.int32, device="cuda")


def _lib():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    return E, rt


def handle(batch, rows, paged=1):
    E, rt = _lib()
    return rt.Handle(E.ebd_config(
        d_model=64, vocab=128, n_heads_q=4, n_heads_kv=4, head_dim=64, d_base=64, max_batch=batch, max_window=1,
        max_rows=rows, max_prefix=0, gen_len=64, g_max=5, l_min=8, l_b=32, eos_id=0, lps_enabled=1, tau=0.9, tau_psi=0.89,
        paged=paged))


class Device:
    """The state of a plan on the device, guarded, and its calls."""

    def __init__(self, ref: Plan, h, rows):
        self.ref, self.h, self.rows = ref, h, rows
        B = len(ref.len)
        self.kv_len = torch.full((B + 2,), 77, **I32)
        self.table = torch.full((B + 2, ref.max_pages), 77, **I32)
        self.free = torch.full((ref.n_pages + 2,), 77, **I32)
        self.n_free = torch.tensor([len(ref.free)], **I32)
        self.cu = torch.full((B + 3,), 77, **I32)
        self.pos = torch.full((rows + 2,), 77, **I32)
        self.slot = torch.full((rows + 2,), 77, dtype=torch.int64, device="cuda")
        self.kv_len[1:-1] = torch.tensor(ref.len, **I32)
        self.table[1:-1] = torch.tensor(ref.table, **I32).view(B, ref.max_pages)
        self.free[1: 1 + len(ref.free)] = torch.tensor(ref.free, **I32)
        self.add = torch.zeros((max(B, 1),), **I32)

    def args(self, outputs=True):
        E, _ = _lib()
        a = E.ebd_paged_plan_args()
        a.batch, a.rows = len(self.ref.len), self.rows if outputs else 0
        a.add, a.kv_len = self.add.data_ptr(), self.kv_len[1:].data_ptr()
        a.page_table, a.free_pages, a.n_free = self.table[1:].data_ptr(), self.free[1:].data_ptr(), self.n_free.data_ptr()
        if outputs:
            a.cu_rows, a.row_pos, a.slot = self.cu[1:].data_ptr(), self.pos[1:].data_ptr(), self.slot[1:].data_ptr()
        a.page_size, a.n_pages, a.max_pages = self.ref.page, self.ref.n_pages, self.ref.max_pages
        return a

    def step(self, add, outputs=True, want=0):
        E, rt = _lib()
        if add:
            self.add.copy_(torch.tensor(add, dtype=torch.int32))
        E.check(E.ebd_paged_plan(self.h.h, self.args(outputs), rt.stream_handle(None)), self.h.h)
        assert self.h.sync_status() == want
        self.check(self.ref.step(add, self.rows if outputs else None), outputs)

    def check(self, rows, outputs):
        r, B = self.ref, len(self.ref.len)
        assert self.kv_len[1:-1].tolist() == r.len
        assert self.table[1:-1].tolist() == r.table
        assert self.n_free.item() == len(r.free) and self.free[1: 1 + len(r.free)].tolist() == r.free
        if outputs:
            cu, pos, slot = rows if rows else ([0] * (B + 1), [], [])
            assert self.cu[1:-1].tolist() == cu
            assert self.pos[1:-1].tolist() == pos + [-1] * (self.rows - len(pos))
            assert self.slot[1:-1].tolist() == slot + [-1] * (self.rows - len(slot))
        for t in (self.kv_len, self.table, self.free, self.cu, self.pos, self.slot):
            assert (t[0] == 77).all() and (t[-1] == 77).all()


@pytest.mark.parametrize("batch,page,max_pages,most", [(1, 16, 4, 20), (3, 16, 9, 40), (64, 64, 5, 60), (1000, 16, 3, 4),
                                                       (1024, 32, 2, 3), (1025, 16, 2, 3), (4096, 256, 2, 1)])
@pytest.mark.parametrize("paged", [0, 1])
def test_plans(batch, page, max_pages, most, paged):
    """Sequences grow, shrink and end, some plans cannot be met."""
    E, _ = _lib()
    rng = random.Random(batch + page)
    n_pages = batch * max_pages * 2 // 3 + 2
    ref = Plan(n_pages, batch, max_pages, page)
    rng.shuffle(ref.free)
    rows = min(4096, batch * most)
    h = handle(batch, rows, paged)
    d = Device(ref, h, rows)
    refused = 0
    for step in range(12):
        add = [rng.choice((0, 1, most, rng.randint(0, most), -rng.randint(1, 2 * most), -(1 << 31) if rng.random() < .1 else 0))
               for _ in range(batch)]
        if step % 4 == 3:
            add = [most] * batch
        probe = Plan(n_pages, batch, max_pages, page)
        probe.len, probe.table, probe.free = list(ref.len), [list(t) for t in ref.table], list(ref.free)
        met = probe.step(add, rows) is not None
        refused += not met
        d.step(add, True, 0 if met else E.EBD_ERR_PAGES)
    d.step([-(1 << 31)] * batch, outputs=False)
    assert sorted(ref.free) == list(range(n_pages))
    h.close()


def test_taking_back_restores_the_stack():
    ref = Plan(500, 40, 12, 16)
    random.Random(1).shuffle(ref.free)
    h = handle(40, 4000)
    d = Device(ref, h, 4000)
    d.step([50 + i for i in range(40)])
    table, free = [list(t) for t in ref.table], list(ref.free)
    add = [i % 7 * 13 for i in range(40)]
    d.step(add)
    d.step([-a for a in add], outputs=False)
    assert ref.table == table and ref.free == free
    h.close()


@pytest.mark.parametrize("batch,pages", [(1, 30000), (3, 9000), (70, 300)])
def test_more_pages_than_a_cta_holds(batch, pages):
    """Whole caches that come and go at once, lengths alone: pages handed out are those
    that other sequences have just given back, and others."""
    ref = Plan(batch * pages + 50, batch, pages, 16)
    random.Random(2).shuffle(ref.free)
    h = handle(batch, 64)
    d = Device(ref, h, 64)
    d.step([16 * pages - 5] * batch, outputs=False)
    half = [(-16 * pages if b % 2 == 0 else 3) for b in range(batch)]
    d.step(half, outputs=False)
    d.step([(16 * pages - 40 if b % 2 == 0 else -16 * pages // 2) for b in range(batch)], outputs=False)
    d.step([b % 2 for b in range(batch)])
    d.step([(-16 * pages if b % 2 == 0 else min(20, 60 // batch)) for b in range(batch)])
    h.close()


def test_no_sequences_and_no_rows():
    ref = Plan(5, 0, 1, 16)
    h = handle(4, 8)
    Device(ref, h, 3).step([])
    ref = Plan(5, 4, 2, 16)
    d = Device(ref, h, 8)
    d.step([0, 0, 0, 0])
    d.step([3, 0, 2, 3])
    d.step([1, 0, 7, 1], want=_lib()[0].EBD_ERR_PAGES)  # nine rows
    h.close()


@pytest.mark.parametrize("kind", range(8))
def test_states_that_do_not_fit(kind):
    """Nothing is written for a state that holds what it cannot."""
    E, rt = _lib()
    ref = Plan(20, 3, 4, 16)
    h = handle(3, 80)
    d = Device(ref, h, 80)
    d.step([20, 5, 40])
    add = [3, 3, 3]
    if kind == 0:
        d.kv_len[2] = -1
    elif kind == 1:
        d.kv_len[2] = 65
    elif kind == 2:
        d.table[1, 1] = -1        # the page that the first new row goes into
    elif kind == 3:
        d.table[2, 0], add = 20, [0, -5, 0]
    elif kind == 4:
        d.n_free.fill_(-1)
    elif kind == 5:
        d.n_free.fill_(21)
    elif kind == 6:
        d.free[1 + len(ref.free) - 1], add = 20, [0, 14, 0]
    else:
        d.n_free.fill_(20)        # pages come back to a full stack
        add = [0, 0, -40]
    names = ("kv_len", "table", "free", "n_free")
    before = {n: getattr(d, n).clone() for n in names}
    d.add.copy_(torch.tensor(add, dtype=torch.int32))
    E.check(E.ebd_paged_plan(h.h, d.args(), rt.stream_handle(None)), h.h)
    assert h.sync_status() == E.EBD_ERR_BOUNDS
    assert all(torch.equal(before[n], getattr(d, n)) for n in names)
    assert d.cu[1:-1].tolist() == [0] * 4 and (d.pos[1:-1] == -1).all() and (d.slot[1:-1] == -1).all()
    h.close()


def test_refused_arguments():
    E, rt = _lib()
    h = handle(3, 64)
    d = Device(Plan(20, 3, 4, 16), h, 64)
    for name, x in (("batch", 4), ("batch", -1), ("rows", 65), ("rows", -1), ("add", 0), ("kv_len", 0), ("page_table", 0),
                    ("free_pages", 0), ("n_free", 0), ("page_size", 15), ("page_size", 48), ("page_size", 512),
                    ("n_pages", 0), ("max_pages", 0)):
        a = d.args()
        setattr(a, name, x)
        assert E.ebd_paged_plan(h.h, a, rt.stream_handle(None)) == E.EBD_ERR_INVALID_ARG, name
    assert E.ebd_paged_plan(None, d.args(), 0) == E.EBD_ERR_INVALID_ARG
    torch.cuda.synchronize()
    h.close()
    h = handle(5000, 64)
    a = d.args()
    a.batch = 4097
    assert E.ebd_paged_plan(h.h, a, rt.stream_handle(None)) == E.EBD_ERR_UNSUPPORTED
    h.close()
