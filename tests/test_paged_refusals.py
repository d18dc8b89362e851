"""What PagedCache's calls refuse before anything is launched (on the CPU: the
library's calls are replaced, no kernel runs)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2609_16450_gb300 import _ebd as E
from paper_2609_16450_gb300 import paged
from paper_2609_16450_gb300 import runtime as rt

HQ, HKV, D = 8, 2, 64


@pytest.fixture
def cache(monkeypatch):
    """A cache whose calls end in a list of (name, q_stride, kv_stride)."""
    calls = []
    for name in ("ebd_paged_write", "ebd_paged_read", "ebd_paged_attention"):
        monkeypatch.setattr(E, name, lambda h, c, a, s, name=name: calls.append((name, a.q_stride, a.kv_stride)) or 0)
    monkeypatch.setattr(E, "check", lambda status, h=None: None)
    monkeypatch.setattr(rt, "stream_handle", lambda stream: 0)
    h = SimpleNamespace(h=None, cfg=SimpleNamespace(n_heads_q=HQ, n_heads_kv=HKV, head_dim=D))
    c = paged.PagedCache(h, n_pages=4, sequences=2, max_pages=2, page_size=16, device="cpu")
    c.calls = calls
    return c


def _ints(*x, device="cpu"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def _rows(n, heads=HKV, device="cpu"):
    return torch.zeros((n, heads, D), dtype=torch.bfloat16, device=device)


def test_dense_and_sliced_rows_are_taken(cache):
    cu, pos = _ints(0, 3), _ints(0, 1, 2)
    fused = torch.zeros((3, HQ + 2 * HKV, D), dtype=torch.bfloat16)
    cache.write(cu, pos, _rows(3), _rows(3))
    cache.write(cu, pos, fused[:, HQ: HQ + HKV], fused[:, HQ + HKV:], skip=torch.zeros(3, dtype=torch.bool))
    cache.read(cu, pos, _rows(3), _rows(3))
    cache.attention(fused[:, :HQ], cu, _ints(3), _rows(3, HQ))
    cache.write(_ints(0, 1), _ints(0), _rows(1).expand(1, HKV, D), _rows(1))
    wide = (HQ + 2 * HKV) * D
    assert cache.calls == [("ebd_paged_write", 0, HKV * D), ("ebd_paged_write", 0, wide), ("ebd_paged_read", 0, HKV * D),
                           ("ebd_paged_attention", wide, 0), ("ebd_paged_write", 0, 0)]


def test_rows_that_overlap_are_refused(cache):
    """A row expanded to several has stride 0, which the C calls take as dense rows."""
    cu, pos = _ints(0, 3), _ints(0, 1, 2)
    for k in (_rows(1).expand(3, HKV, D), torch.zeros(4096, dtype=torch.bfloat16).as_strided((3, HKV, D), (D, D, 1))):
        for call in (cache.write, cache.read):
            with pytest.raises(ValueError, match="overlap"):
                call(cu, pos, k, k)
    q = _rows(1, HQ).expand(3, HQ, D)
    with pytest.raises(ValueError, match="overlap"):
        cache.attention(q, cu, _ints(3), _rows(3, HQ))
    assert not cache.calls


def test_tensors_of_another_device_are_refused(cache):
    here = dict(cu_rows=_ints(0, 3), row_pos=_ints(0, 1, 2), k=_rows(3), v=_rows(3))
    for what in here:
        args = dict(here, **{what: here[what].to("meta")})
        for call in (cache.write, cache.read):
            with pytest.raises(ValueError, match=what):
                call(**args)
    with pytest.raises(ValueError, match="skip"):
        cache.write(**here, skip=torch.zeros(3, dtype=torch.uint8, device="meta"))
    here = dict(q=_rows(3, HQ), cu_rows=_ints(0, 3), kv_len=_ints(3), out=_rows(3, HQ))
    for what in here:
        with pytest.raises(ValueError, match=what):
            cache.attention(**dict(here, **{what: here[what].to("meta")}))
    assert not cache.calls


def test_lengths_below_zero_are_refused():
    """A negative length would put the table's empty entries among the free pages."""
    t = paged.PageTable(8, 2, 5, 16)
    t.reserve(0, 20)
    for call in (t.reserve, t.release):
        for length in (-1, -16, -40):
            with pytest.raises(ValueError, match="length"):
                call(0, length)
    assert t.release(0) and sorted(t._free) == list(range(8))
