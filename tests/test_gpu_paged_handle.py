"""Handles of ebd_config.paged = 1: one that only pages takes only what paging
needs; the decoding step is set up when it is first used, and is as ever."""
import numpy as np
import pytest

import synth
from tests import paged_ref as pr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _lib():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    return E, rt


def _free():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]


def test_a_handle_that_pages_takes_its_own_workspace_alone():
    E, rt = _lib()
    pr.handle(E, rt, (4, 4, 128), 1, 1).close()  # the context's own memory
    cfg = lambda paged: E.ebd_config(  # noqa: E731
        d_model=4096, vocab=1000000, n_heads_q=32, n_heads_kv=32, head_dim=128, d_base=4096, max_batch=64, max_window=64,
        max_rows=4096, max_prefix=8192, gen_len=64, g_max=5, l_min=8, l_b=32, eos_id=63, lps_enabled=1, tau=0.9,
        tau_psi=0.89, paged=paged)
    taken = []
    for paged in (1, 0):
        before = _free()
        h = rt.Handle(cfg(paged))
        taken.append(before - _free())
        h.close()
    # 2 x 152 tiles of 256 rows of 130 floats, and records; the token table alone is 256 MB
    assert taken[0] < 64 << 20 and taken[1] > 256 << 20


def _handles(sh):
    E, rt = _lib()
    inp = synth.make_step_inputs(sh)
    w = rt.upload_weights(inp)
    return E, rt, inp, w, rt.Handle(rt.config_for(sh), w.w_emb), rt.Handle(rt.config_for(sh, paged=1))


@pytest.mark.parametrize("first", ["bind", "lm_stats", "attention", "export", "import"])
def test_the_step_of_a_handle_that_pages(first):
    """The same results as another handle's, whichever function comes first."""
    sh = synth.tiny
    E, rt, inp, w, h, hp = _handles(sh)
    outs, blob = [], E.ebd_export_weights(h.h)[1]
    for g in (h, hp):
        ds = rt.DeviceStep(inp, w)
        if g is hp and first == "lm_stats":
            E.check(E.ebd_lm_stats(g.h, ds.args(), rt.stream_handle(None)), g.h)
        if g is hp and first == "attention":
            E.check(E.ebd_attention(g.h, ds.args(), rt.stream_handle(None)), g.h)
        if g is hp and first == "export":
            np.testing.assert_array_equal(E.ebd_export_weights(hp.h)[1], blob)
        if g is hp and first == "import":
            assert E.ebd_import_weights(hp.h, blob) == 0
        if g is hp:
            assert E.ebd_step(g.h, ds.args(), rt.stream_handle(None)) == E.EBD_ERR_STATE
            g.bind(w.w_emb)
            np.testing.assert_array_equal(E.ebd_export_weights(hp.h)[1], blob)
        E.check(E.ebd_step(g.h, ds.args(), rt.stream_handle(None)), g.h)
        assert g.sync_status() == 0
        outs.append(ds.fetch())
        g.close()
    for k in outs[0]:
        np.testing.assert_array_equal(outs[0][k], outs[1][k], err_msg=k)


def test_the_first_decoding_call_is_refused_in_a_capture():
    E, rt, inp, w, h, hp = _handles(synth.tiny)
    ds = rt.DeviceStep(inp, w)
    graph = torch.cuda.CUDAGraph()
    keep = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        keep.add_(1)
        status = E.ebd_lm_stats(hp.h, ds.args(), rt.stream_handle(None))
    assert status == E.EBD_ERR_STATE and "capture" in E.ebd_last_error(hp.h)
    E.check(E.ebd_lm_stats(hp.h, ds.args(), rt.stream_handle(None)), hp.h)
    assert hp.sync_status() == 0
    h.close(), hp.close()
