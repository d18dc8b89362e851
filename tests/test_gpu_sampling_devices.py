"""Host tensors are refused by a real handle's calls."""
import pytest

from tests.test_gpu_sample import handle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_host_tensors():
    from paper_2609_16450_gb300 import sampling as sp
    from paper_2609_16450_gb300.paged import PagedCache
    h = handle(100, 8)
    assert h.device == torch.zeros(1, device="cuda").device
    logits, u = torch.zeros((8, 100)), torch.zeros(8)
    with pytest.raises(ValueError):
        sp.sample(h, logits, u, torch.zeros(8, dtype=torch.int32), u)
    with pytest.raises(ValueError):
        PagedCache(h, n_pages=6, sequences=3, max_pages=2, page_size=16, device="cpu", plan="device")
    token, prob = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda")
    sp.sample(h, logits.cuda(), u.cuda(), token, prob)
    assert h.sync_status() == 0 and (token == 0).all()
    h.close()
