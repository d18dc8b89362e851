"""ebd_lm_logits: logits in memory, and the statistics beside them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _lib():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    return E, rt


def handle(d, vocab, rows):
    E, rt = _lib()
    return rt.Handle(E.ebd_config(
        d_model=d, vocab=vocab, n_heads_q=4, n_heads_kv=4, head_dim=64, d_base=64, max_batch=rows, max_window=min(rows, 64),
        max_rows=rows, max_prefix=0, gen_len=64, g_max=5, l_min=8, l_b=32, eos_id=0, lps_enabled=1, tau=0.9, tau_psi=0.89))


def inputs(d, vocab, rows, packed, h):
    _, rt = _lib()
    g = torch.Generator(device="cuda").manual_seed(d + vocab + rows)
    x = torch.randn((rows, d), generator=g, device="cuda").bfloat16()
    w = (torch.randn((vocab, d), generator=g, device="cuda") / d ** 0.5).bfloat16()
    held = rt.DeviceWeights(w_lm=w, w_emb=None)
    return x, w, rt.pack_weights(h, held) if packed else held


def args(x, w):
    E, _ = _lib()
    a = E.ebd_step_args()
    a.batch = a.rows = x.shape[0]
    a.hidden, a.w_lm, a.w_lm_layout = x.data_ptr(), w.w_lm.data_ptr(), w.layout
    return a


@pytest.mark.parametrize("packed", [0, 1])
@pytest.mark.parametrize("rows,d,vocab,pad", [(1, 64, 130, 0), (7, 256, 4096, 1), (32, 1032, 1001, 0), (64, 512, 20011, 64),
                                              (65, 512, 20011, 3), (129, 72, 7001, 0), (257, 512, 10007, 1),
                                              (300, 136, 30000, 9), (512, 256, 4096, 0), (700, 128, 3001, 5)])
def test_logits(rows, d, vocab, pad, packed):
    """Sums of d products in 32 bits: off by at most d 2^-23 of the sum of their
    magnitudes, every addition cut by less than a step (tensor cores need not round)."""
    E, rt = _lib()
    h = handle(d, vocab, rows)
    x, w, held = inputs(d, vocab, rows, packed, h)
    out = torch.full((rows + 2, vocab + pad), 7.0, device="cuda")
    E.check(E.ebd_lm_logits(h.h, args(x, held), out[1].data_ptr(), out.stride(0), rt.stream_handle(None)), h.h)
    assert h.sync_status() == 0
    want = x.double() @ w.double().T
    most = (x.double().abs() @ w.double().abs().T) * (d * 2.0 ** -23)
    assert ((out[1:-1, :vocab].double() - want).abs() <= most).all()
    assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[1:-1, vocab:] == 7).all()
    h.close()


@pytest.mark.parametrize("rows,d", [(5, 256), (64, 1032), (130, 1536), (300, 2056), (512, 640)])
def test_statistics_beside_the_logits(rows, d):
    """They are the stored logits', as ebd_lm_stats computes them from its own: in 32 bits,
    by fast exponentials (off by 2^-21 each and in their sums, what the entropy weighs
    with |l - m| < 64 at most).  The logits do not depend on them."""
    E, rt = _lib()
    vocab = 4096
    h = handle(d, vocab, rows)
    x, w, held = inputs(d, vocab, rows, 1, h)
    names = ("conf", "entropy", "ent_norm", "gap", "argmax")
    t = {n: torch.zeros(rows, dtype=torch.int32 if n == "argmax" else torch.float32, device="cuda") for n in names}
    outs = [torch.full((rows, vocab), 7.0, device="cuda") for _ in range(2)]
    for call in range(2):
        a = args(x, held)
        if call == 0:
            for n in names:
                setattr(a, n, t[n].data_ptr())
        E.check(E.ebd_lm_logits(h.h, a, outs[call].data_ptr(), 0, rt.stream_handle(None)), h.h)
    assert h.sync_status() == 0
    l = outs[0].double()
    p = torch.softmax(l, 1)
    top = l.topk(2, 1).values
    want = dict(conf=p.max(1).values, entropy=-(p * p.log()).sum(1), gap=p.max(1).values - torch.exp(top[:, 1] - torch.logsumexp(l, 1)))
    want["ent_norm"] = want["entropy"] / np.log(vocab)
    for n, v in want.items():
        assert ((t[n].double() - v).abs() <= 64 * 2.0 ** -20).all(), n
    assert torch.equal(outs[0].argmax(1).int(), t["argmax"])
    assert torch.equal(outs[0], outs[1])
    h.close()


@pytest.mark.parametrize("rows", [32, 200])
def test_long_sums(rows):
    """4096 columns: no worse than sums of 1024 rounded down at every step and added, whose
    error is at most 64 cuts of a partial sum (16 columns each) by 2^-23 and 4 roundings."""
    E, rt = _lib()
    d, vocab = 4096, 3000
    h = handle(d, vocab, rows)
    x, w, held = inputs(d, vocab, rows, 1, h)
    out = torch.zeros((rows, vocab), device="cuda")
    E.check(E.ebd_lm_logits(h.h, args(x, held), out.data_ptr(), 0, rt.stream_handle(None)), h.h)
    assert h.sync_status() == 0
    p = x.double()[:, None].view(rows, 1, 4, 1024) * w.double()[None].view(1, vocab, 4, 1024)[:, :500]
    most = (p.abs().sum(3) * 64 * 2.0 ** -23).sum(2) + p.abs().sum((2, 3)) * 4 * 2.0 ** -24
    assert ((out[:, :500].double() - p.sum((2, 3))).abs() <= most).all()
    # and as a rule far better: a cut is of a partial sum, which is no larger than the
    # segment's, a half of the logits as these go; the segments' errors add up as their sums do
    rms = (out[:, :500].double() - p.sum((2, 3))).square().mean().sqrt() / p.sum((2, 3)).square().mean().sqrt()
    assert rms < 64 * 2.0 ** -23 + 4 * 2.0 ** -24
    h.close()


def test_refusals():
    E, rt = _lib()
    h = handle(64, 100, 8)
    x, w, held = inputs(64, 100, 8, 0, h)
    out = torch.zeros((8, 100), device="cuda")
    call = lambda a, p, s: E.ebd_lm_logits(h.h, a, p, s, rt.stream_handle(None))  # noqa: E731
    assert call(args(x, held), 0, 0) == E.EBD_ERR_INVALID_ARG
    assert call(args(x, held), out.data_ptr() + 2, 0) == E.EBD_ERR_INVALID_ARG
    assert call(args(x, held), out.data_ptr(), 99) == E.EBD_ERR_INVALID_ARG
    a = args(x, held)
    a.rows = a.batch = 9
    assert call(a, out.data_ptr(), 0) == E.EBD_ERR_INVALID_ARG
    a.rows = a.batch = 0
    assert call(a, 0, 0) == E.EBD_OK
    a = args(x, held)
    a.w_lm = 0
    assert call(a, out.data_ptr(), 0) == E.EBD_ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert (out == 0).all()
    h.close()
