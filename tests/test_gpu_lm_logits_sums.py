"""ebd_lm_logits: what its sums are off by, and what they do not depend on."""
import pytest

from tests.test_gpu_lm_logits import _lib, args, handle, inputs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def logits_of(h, x, held, vocab, stats=()):
    E, rt = _lib()
    rows = x.shape[0]
    a = args(x, held)
    t = {n: torch.zeros(rows, dtype=torch.int32 if n == "argmax" else torch.float32, device="cuda") for n in stats}
    for n in t:
        setattr(a, n, t[n].data_ptr())
    out = torch.full((rows, vocab), 7.0, device="cuda")
    E.check(E.ebd_lm_logits(h.h, a, out.data_ptr(), 0, rt.stream_handle(None)), h.h)
    assert h.sync_status() == 0
    return out


@pytest.mark.parametrize("packed", [0, 1])
@pytest.mark.parametrize("d", [72, 328, 1032, 4096])
@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 40, 48, 49, 64, 65, 96, 97, 200, 256, 257, 400])
def test_statistics_leave_the_logits_alone(rows, d, packed):
    """Bit for bit: their buffers leave the sums their segments."""
    vocab = 1000
    h = handle(d, vocab, rows)
    x, _, held = inputs(d, vocab, rows, packed, h)
    alone = logits_of(h, x, held, vocab)
    assert torch.equal(alone, logits_of(h, x, held, vocab, ("conf", "entropy", "ent_norm", "gap", "argmax")))
    assert torch.equal(alone, logits_of(h, x, held, vocab, ("argmax",)))
    h.close()
