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


@pytest.mark.parametrize("rows", [5, 64, 130, 300])
def test_statistics_beside_the_logits_are_ebd_lm_stats(rows):
    """The same kernel path: bit for bit; and logits do not depend on them."""
    E, rt = _lib()
    d, vocab = 256, 4096
    h = handle(d, vocab, rows)
    x, w, held = inputs(d, vocab, rows, 1, h)
    names = ("conf", "entropy", "ent_norm", "gap", "argmax")
    got = []
    outs = [torch.full((rows, vocab), 7.0, device="cuda") for _ in range(2)]
    for call in range(3):
        a = args(x, held)
        t = {n: torch.zeros(rows, dtype=torch.int32 if n == "argmax" else torch.float32, device="cuda") for n in names}
        if call < 2:
            for n in names:
                setattr(a, n, t[n].data_ptr())
        if call == 0:
            E.check(E.ebd_lm_stats(h.h, a, rt.stream_handle(None)), h.h)
        else:
            E.check(E.ebd_lm_logits(h.h, a, outs[call - 1].data_ptr(), 0, rt.stream_handle(None)), h.h)
        got.append(t)
    assert h.sync_status() == 0
    for n in names:
        assert torch.equal(got[0][n], got[1][n]), n
    assert torch.equal(outs[0], outs[1])
    assert torch.equal(outs[0].argmax(1).int(), got[0]["argmax"])
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
