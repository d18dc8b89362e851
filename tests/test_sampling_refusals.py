"""What the sampling functions and plans on the device refuse before anything is
launched (on the CPU: the library's calls are replaced, no kernel runs)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2609_16450_gb300 import _ebd as E
from paper_2609_16450_gb300 import paged
from paper_2609_16450_gb300 import runtime as rt
from paper_2609_16450_gb300 import sampling as sp

D, V, R = 64, 100, 4


@pytest.fixture
def lib(monkeypatch):
    """A handle, and the arguments of the calls that are reached."""
    calls = []
    monkeypatch.setattr(E, "ebd_lm_logits", lambda h, a, p, s, st: calls.append((a, p, s)) or 0)
    monkeypatch.setattr(E, "ebd_sample", lambda h, a, st: calls.append(a) or 0)
    monkeypatch.setattr(E, "ebd_paged_plan", lambda h, a, st: calls.append(a) or 0)
    monkeypatch.setattr(E, "check", lambda status, h=None: None)
    monkeypatch.setattr(rt, "stream_handle", lambda stream: 0)
    cfg = SimpleNamespace(d_model=D, vocab=V, max_batch=R, n_heads_q=8, n_heads_kv=2, head_dim=64)
    return SimpleNamespace(h=SimpleNamespace(h=None, cfg=cfg), calls=calls)


def _w():
    return rt.DeviceWeights(w_lm=torch.zeros((V, D), dtype=torch.bfloat16), w_emb=None)


def test_logits(lib):
    x, out = torch.zeros((R, D), dtype=torch.bfloat16), torch.zeros((R, V + 3))
    stats = {n: torch.zeros(R, dtype=t) for n, t in sp.STATS.items()}
    sp.lm_logits(lib.h, x, _w(), out[:, :V], stats)
    sp.lm_logits(lib.h, x.view(torch.int16), _w(), torch.zeros((R, V)))
    sp.lm_logits(lib.h, x[:1], _w(), out[:1, :V])
    assert [c[2] for c in lib.calls] == [V + 3, V, 0] and lib.calls[0][0].conf == stats["conf"].data_ptr()
    for bad in (dict(hidden=x.float()), dict(hidden=x[:, :D - 1]), dict(hidden=torch.zeros((D, R), dtype=torch.bfloat16).T),
                dict(hidden=x[:3]), dict(hidden=x.to("meta")), dict(logits=out), dict(logits=out[:, :V].double()),
                dict(logits=out[:, :V].to("meta")), dict(logits=torch.zeros((V, R)).T),
                dict(logits=torch.zeros((1, V)).expand(R, V)), dict(stats={"mean": out}),
                dict(stats={"conf": torch.zeros(R + 1)}), dict(stats={"argmax": torch.zeros(R)}),
                dict(stats={"gap": torch.zeros(R, device="meta")})):
        args = dict(dict(hidden=x, logits=out[:, :V], stats=None), **bad)
        with pytest.raises(ValueError):
            sp.lm_logits(lib.h, args["hidden"], _w(), args["logits"], args["stats"])
    assert len(lib.calls) == 3


def test_sample(lib):
    ok = dict(logits=torch.zeros((R, V)), u=torch.zeros(R), token=torch.zeros(R, dtype=torch.int32), prob=torch.zeros(R),
              temperature=torch.ones(R), top_k=torch.zeros(R, dtype=torch.int32), top_p=torch.ones(R), min_p=torch.zeros(R))
    sp.sample(lib.h, **ok)
    for t, code in ((torch.bfloat16, E.EBD_LOGITS_BF16), (torch.float16, E.EBD_LOGITS_F16)):
        sp.sample(lib.h, **dict(ok, logits=torch.zeros((R, V + 1), dtype=t)[:, :V], top_k=None))
        assert lib.calls[-1].dtype == code and lib.calls[-1].stride == V + 1 and not lib.calls[-1].top_k
    n = len(lib.calls)
    for name, t in ok.items():
        if name == "logits":
            bads = (t.double(), t[:, 1:], torch.zeros((V, R)).T, torch.zeros((1, V)).expand(R, V), t[0])
        else:
            bads = (t[:3], t.double(), torch.zeros(2 * R, dtype=t.dtype)[::2], t.to("meta"), t.view(R, 1))
        for bad in bads:
            with pytest.raises(ValueError):
                sp.sample(lib.h, **dict(ok, **{name: bad}))
    assert len(lib.calls) == n


def test_settings():
    assert sp.Settings().rows(3, "cpu")["top_k"] is None
    r = sp.Settings(0.5, 7, 0.9, 0.1).rows(3, "cpu")
    assert r["top_k"].dtype == torch.int32 and [float(r[k][2]) for k in ("temperature", "top_k")] == [0.5, 7.0]
    assert set(r) == {"temperature", "top_k", "top_p", "min_p"}


def test_plans(lib):
    make = lambda plan: paged.PagedCache(lib.h, n_pages=6, sequences=3, max_pages=2, page_size=16, device="cpu", plan=plan)  # noqa: E731
    with pytest.raises(ValueError):
        make("gpu")
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    host, c = make("host"), make("device")
    with pytest.raises(RuntimeError):
        host.plan(i32(3))
    for call in (c.reserve, c.release):
        with pytest.raises(RuntimeError):
            call(0, 5)
    c.plan(i32(3))
    c.plan(i32(2), i32(3), i32(7), torch.zeros(7, dtype=torch.int64))
    assert [a.rows for a in lib.calls] == [0, 7] and lib.calls[1].batch == 2
    for bad in (dict(add=i32(4)), dict(add=i32(3).long()), dict(add=i32(6)[::2]), dict(add=i32(3).to("meta")),
                dict(cu_rows=i32(3)), dict(cu_rows=i32(4).long()), dict(row_pos=i32(3).float()),
                dict(row_pos=i32(3), slot=torch.zeros(4, dtype=torch.int64)), dict(slot=i32(3)),
                dict(slot=torch.zeros(3, dtype=torch.int64, device="meta"))):
        with pytest.raises(ValueError):
            c.plan(**dict(dict(add=i32(3)), **bad))
    assert len(lib.calls) == 2
