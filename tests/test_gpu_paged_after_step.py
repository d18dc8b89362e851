"""A step, then a paged write of the rows it has committed, on one stream: the
write's mask is what the decision writes, while the window attention, launched
between them, does not wait for the decision to do its own work."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("shape", [
    synth.tiny.with_(prefix=0, windows=(64,)),
    synth.tiny.with_(batch=3, prefix=16, windows=(64, 5, 33), seed=4),
    synth.tiny.with_(batch=40, prefix=0, windows=(16,) * 40, seed=5),
    synth.tiny.with_(d_model=1024, vocab=32000, n_heads_q=8, n_heads_kv=4, head_dim=128, windows=(64,), seed=6),
], ids=["one", "ragged", "many", "wide"])
def test_rows_committed_by_the_step_before(shape, dtype):
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    from paper_2609_16450_gb300.paged import PagedCache
    from tests import paged_ref as pr
    inp = synth.make_step_inputs(shape)
    w = rt.upload_weights(inp)
    h = rt.Handle(rt.config_for(shape), w.w_emb)
    ds = rt.DeviceStep(inp, w)
    B, R, H, D = shape.batch, inp.rows, shape.n_heads_kv, shape.head_dim
    need = (int(inp.row_pos.max()) + 16) // 16
    c = PagedCache(h, B * need, B, need, 16, dtype)
    for b in range(B):
        c.reserve(b, 16 * need)
    k, v = (x.view(torch.bfloat16).view(R, H, D) for x in (ds.k_win, ds.v_win))
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    seen = set()
    for trial in range(25):
        c.k.zero_(), c.v.zero_()
        if c.k_scale is not None:
            c.k_scale.zero_(), c.v_scale.zero_()
        ds.restore_state()
        E.check(E.ebd_step(h.h, ds.args(), rt.stream_handle(None)), h.h)
        c.write(ds.cu_rows, ds.row_pos, k, v, skip=ds.mask)
        c.read(ds.cu_rows, ds.row_pos, kb, vb)
        assert h.sync_status() == 0
        kept = ds.mask == 0
        seen.add(int(kept.sum()))
        for got, rows in ((kb, k), (vb, v)):
            want = rows.double().cpu().numpy()
            if dtype == "e4m3":
                want = pr.dequantise(*pr.quantise(want))
            want = np.where(kept.cpu().numpy()[:, None, None], want, 0.0)
            np.testing.assert_array_equal(got.double().cpu().numpy(), want)
    before = int((ds.state0[1] == 0).sum())
    assert len(seen) == 1 and seen.pop() > before  # the step committed rows
    h.close()
