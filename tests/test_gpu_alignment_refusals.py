"""Buffers that are not aligned to what they hold are refused before anything is launched."""
import pytest

from tests.test_gpu_sample import handle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_sample():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    h = handle(100, 8)
    t, v = torch.zeros((9, 100), device="cuda"), torch.zeros(16, device="cuda")
    names = ("u", "temperature", "top_k", "top_p", "min_p", "token", "prob")
    for name in names:
        for off in (1, 2, 3):
            a = E.ebd_sample_args()
            a.rows, a.logits = 8, t.data_ptr()
            for n in names:
                setattr(a, n, v.data_ptr() + (off if n == name else 0))
            assert E.ebd_sample(h.h, a, rt.stream_handle(None)) == E.EBD_ERR_INVALID_ARG, (name, off)
    torch.cuda.synchronize()
    assert (v == 0).all() and h.sync_status() == 0
    h.close()


def test_plan():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    h = handle(100, 8)
    v = torch.zeros(256, dtype=torch.int64, device="cuda")
    names = ("add", "kv_len", "page_table", "free_pages", "n_free", "cu_rows", "row_pos", "slot")
    for name in names:
        for off in (1, 2, 3) + ((4,) if name == "slot" else ()):
            a = E.ebd_paged_plan_args()
            a.batch, a.rows, a.page_size, a.n_pages, a.max_pages = 2, 4, 16, 8, 4
            for i, n in enumerate(names):
                setattr(a, n, v.data_ptr() + 128 * i + (off if n == name else 0))
            assert E.ebd_paged_plan(h.h, a, rt.stream_handle(None)) == E.EBD_ERR_INVALID_ARG, (name, off)
    torch.cuda.synchronize()
    assert (v == 0).all() and h.sync_status() == 0
    h.close()
