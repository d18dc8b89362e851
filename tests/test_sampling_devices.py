"""Tensors that a handle's kernels cannot read are refused before anything is launched, also
where all of a call's are on one device (on the CPU: the library's calls are replaced)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2609_16450_gb300 import _ebd as E
from paper_2609_16450_gb300 import paged
from paper_2609_16450_gb300 import runtime as rt
from paper_2609_16450_gb300 import sampling as sp

D, V, R = 64, 100, 4


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_tensors_of_another_device_than_the_handle(device, monkeypatch):
    calls = []
    for name in ("ebd_lm_logits", "ebd_sample", "ebd_paged_plan"):
        monkeypatch.setattr(E, name, lambda *a: calls.append(a) or 0)
    monkeypatch.setattr(E, "check", lambda status, h=None: None)
    monkeypatch.setattr(rt, "stream_handle", lambda stream: 0)
    cfg = SimpleNamespace(d_model=D, vocab=V, max_batch=R, n_heads_q=8, n_heads_kv=2, head_dim=64)
    h = SimpleNamespace(h=None, cfg=cfg, device=torch.device("cuda", 0))
    x = torch.zeros((R, D), dtype=torch.bfloat16, device=device)
    w = rt.DeviceWeights(w_lm=torch.zeros((V, D), dtype=torch.bfloat16, device=device), w_emb=None)
    logits, v = torch.zeros((R, V), device=device), torch.zeros(R, device=device)
    with pytest.raises(ValueError, match="the handle on cuda:0"):
        sp.lm_logits(h, x, w, logits)
    with pytest.raises(ValueError, match="the handle on cuda:0"):
        sp.sample(h, logits, v, torch.zeros(R, dtype=torch.int32, device=device), v)
    for plan in ("host", "device"):
        with pytest.raises(ValueError, match="the handle on cuda:0"):
            paged.PagedCache(h, n_pages=6, sequences=3, max_pages=2, page_size=16, device=device, plan=plan)
    assert not calls
    h.device = torch.device(device)
    sp.sample(h, logits, v, torch.zeros(R, dtype=torch.int32, device=device), v)
    assert len(calls) == 1
