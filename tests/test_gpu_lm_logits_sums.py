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


@pytest.mark.parametrize("rows,vocab", [(1, 3000), (24, 3000), (32, 3000), (40, 3000), (64, 3000), (65, 3000), (200, 3000),
                                        (256, 3000), (300, 3000), (512, 3000)])
def test_no_worse_than_plain_sums(rows, vocab):
    """4096 columns, against the plain sum in 32 bits: one product after the other, every
    addition rounded.  Errors as a rule (their rms) are no larger than that sum's; columns
    that all went into one accumulator would be off by six times as much."""
    d, look = 4096, 500
    h = handle(d, vocab, rows)
    x, w, held = inputs(d, vocab, rows, 1, h)
    out = logits_of(h, x, held, vocab)
    xs, ws = x.float(), w[-look:].float()
    plain = torch.zeros((rows, min(look, vocab)), device="cuda")
    for k in range(d):
        plain.addcmul_(xs[:, k: k + 1], ws[:, k][None])
    want = x.double() @ w[-look:].double().T
    rms = lambda t: (t.double() - want).square().mean().sqrt()  # noqa: E731
    assert rms(out[:, -look:]) <= rms(plain), (float(rms(out[:, -look:])), float(rms(plain)))
    h.close()


@pytest.mark.parametrize("rows,d", [(200, 640), (200, 648), (200, 768), (130, 1032), (300, 1536), (200, 2056), (512, 2600)])
def test_segments_of_any_number(rows, d):
    """Sums of other numbers of columns, cut into segments that end within a stage or are
    one: every addition cut by less than a step, and added to no other row's."""
    vocab = 700
    h = handle(d, vocab, rows)
    x, w, held = inputs(d, vocab, rows, 1, h)
    out = logits_of(h, x, held, vocab)
    want = x.double() @ w.double().T
    most = (x.double().abs() @ w.double().abs().T) * (d * 2.0 ** -23)
    assert ((out.double() - want).abs() <= most).all()
    h.close()
