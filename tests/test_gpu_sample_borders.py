"""ebd_sample where its borders are hardest to find: shares close to 1."""
import numpy as np
import pytest

from tests.test_gpu_sample import handle, make, sample, verify

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LAST = np.float32(1 - 2.0 ** -24)  # the last number below 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,rows", [(500, 24), (4096, 24), (4096, 200), (152064, 12), (152064, 90)])
def test_top_p_near_one(vocab, rows, dtype):
    """The share that is left out lies below all roundings of what bounds the sums by
    bins (10^-4): by itself, and of what top-k leaves."""
    h = handle(vocab)
    logits, g = make(rows, vocab, dtype, seed=vocab + rows)
    p = np.resize(np.array([0.9999, 0.99995, 0.99999, LAST], np.float32), rows)
    u = g.uniform(0, 1, rows).astype(np.float32) * LAST
    u[::3] = LAST
    T = np.exp(g.uniform(np.log(0.3), np.log(2), rows)).astype(np.float32)
    for k in (None, np.full(rows, vocab * 4 // 5, np.int32), np.full(rows, vocab // 40, np.int32)):
        for t in (None, T):
            token, prob, status = sample(h, logits, u, t, k, p)
            assert status == 0
            verify(logits, t, k, p, None, u, token, prob)
    h.close()
