"""Logits, sampling and plans on the device as they are used together: in the
generation loop, and as one captured step of a server."""
import numpy as np
import pytest

import synth
from oracle import ebd_oracle as o
from tests import paged_ref as pr
from tests import parity
from tests import sample_ref
from tests.plan_ref import Plan

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _loop(sh, paged=False, **opts):
    from paper_2609_16450_gb300 import loop as lp
    from paper_2609_16450_gb300 import runtime as rt
    inp = synth.make_step_inputs(sh)
    w = rt.upload_weights(inp)
    h = rt.Handle(lp.config_for_loop(sh, paged=int(paged)), w.w_emb)
    try:
        return lp.run_loop(h, sh, w, lambda s, p: synth.loop_window_inputs(sh, s, p), lambda p: synth.loop_kv(sh, p),
                           cache="paged" if paged else "prefix", **opts)
    finally:
        h.close()


def _uniforms(step, positions):
    return np.random.default_rng(step * 7919 + int(positions[0])).random(len(positions)).astype(np.float32) * np.float32(
        1 - 2.0 ** -24)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("e4m3", 64)])
def test_loop_with_plans_on_the_device(dtype, page):
    """What it is with plans on the host, bit for bit."""
    host, dev = (_loop(synth.loop_tiny, paged=True, kv_dtype=dtype, page_size=page, plan=p) for p in ("host", "device"))
    assert host.commits == dev.commits and np.array_equal(host.tokens, dev.tokens)
    for a, b in zip(host.records, dev.records):
        assert a.window == b.window and np.array_equal(a.attn_out, b.attn_out)
    n = synth.loop_tiny.prefix + max(r.window[1] for r in host.records)
    assert np.array_equal(host.k_cache[:n], dev.k_cache[:n]) and np.array_equal(host.v_cache[:n], dev.v_cache[:n])


@pytest.mark.parametrize("settings", [dict(temperature=0.7, top_k=50, top_p=0.9), dict(temperature=1.3, min_p=0.05),
                                      dict(temperature=0.0)])
def test_sampling_loop(settings):
    """Every x_hat and kappa is what the step's logits and numbers give, and every
    decision follows from them by the rules."""
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import loop as lp
    from paper_2609_16450_gb300 import runtime as rt
    from paper_2609_16450_gb300 import sampling as sp
    sh = synth.loop_tiny
    res = _loop(sh, sampling=sp.Settings(**settings), uniforms=_uniforms)
    assert sum(res.commits) == sh.gen_len and all(c >= 1 for c in res.commits)
    assert ((0 <= res.tokens) & (res.tokens < sh.vocab)).all()
    w = rt.upload_weights(synth.make_step_inputs(sh))
    h = rt.Handle(lp.config_for_loop(sh), w.w_emb)
    prm = o.DecisionParams(tau=sh.tau, tau_psi=sh.tau_psi, l_min=sh.l_min, l_b=sh.l_b, g_max=sh.g_max, eos_id=sh.eos_id,
                           lps_enabled=bool(sh.lps_enabled))
    plain = _loop(sh)
    for r in res.records:
        lo, hi = r.window
        pos = (sh.prefix + np.arange(lo, hi)).astype(np.int32)
        hid = rt._dev(synth.loop_window_inputs(sh, r.step, pos)[0], "cuda").view(hi - lo, -1)
        logits = torch.empty((hi - lo, sh.vocab), device="cuda")
        sp.lm_logits(h, hid, w, logits)
        l, u = logits.cpu().numpy(), _uniforms(r.step, pos)
        for i in range(hi - lo):
            sample_ref.check(l[i], settings["temperature"], u[i], r.argmax[i], r.conf[i], settings.get("top_k", 0),
                             settings.get("top_p", 1.0), settings.get("min_p", 0.0))
        b = r.before
        out = {"conf": r.conf, "argmax": r.argmax, "lbs_logit": r.lbs_logit, "lps_prob": r.lps_prob, "accepted": r.accepted,
               "tokens": r.after["tokens"], "mask": r.after["mask"], "in_block": r.after["in_block"]}
        parity.check_decision_valid(pos, b["mask"], b["tokens"], b["in_block"], b["meta"], out, r.after["meta"], prm)
    # the statistics beside the logits are those of the plain step
    for a, b in zip(res.records[:1], plain.records[:1]):
        for k in ("entropy", "ent_norm", "gap"):
            parity._close(k, getattr(a, k), getattr(b, k))
    assert h.sync_status() == E.EBD_OK
    h.close()


def test_sampling_in_the_other_settings():
    """The full sequence as the window, the paged cache planned on the device, and the
    baselines' rules, all by drawn tokens."""
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import loop as lp
    from paper_2609_16450_gb300 import runtime as rt
    from paper_2609_16450_gb300 import sampling as sp
    draw = dict(sampling=sp.Settings(0.8, top_p=0.9), uniforms=_uniforms)
    res = _loop(synth.loop_tiny, paged=True, plan="device", **draw)
    plain = _loop(synth.loop_tiny, **draw)
    assert np.array_equal(res.tokens, plain.tokens) and res.commits == plain.commits
    sh = synth.loop_full_tiny
    w = rt.upload_weights(synth.make_step_inputs(sh))
    inputs = (lambda s, p: synth.loop_window_inputs(sh, s, p), lambda p: synth.loop_kv(sh, p))
    h = rt.Handle(lp.config_for_loop(sh, max_window=sh.gen_len), w.w_emb)
    res = lp.run_loop(h, sh, w, *inputs, attention=False, window="full", max_steps=6, **draw)
    assert all(c >= 1 for c in res.commits)
    for r in res.records:
        acc = r.accepted.astype(bool)
        assert np.array_equal(r.after["tokens"][acc], r.argmax[acc])
    h.close()
    sh = synth.loop_tiny
    w = rt.upload_weights(synth.make_step_inputs(sh))
    inputs = (lambda s, p: synth.loop_window_inputs(sh, s, p), lambda p: synth.loop_kv(sh, p))
    for mode in (E.EBD_DECODE_THRESHOLD, E.EBD_DECODE_TOPM):
        h = rt.Handle(lp.config_for_loop(sh, decode_mode=mode, top_m=3), w.w_emb)
        res = lp.run_loop(h, sh, w, *inputs, **draw)
        assert sum(res.commits) == sh.gen_len and ((res.tokens >= 0) & (res.tokens < sh.vocab)).all()
        h.close()


def test_loop_refusals():
    from paper_2609_16450_gb300 import sampling as sp
    for bad in (dict(plan="device"), dict(plan="gpu"), dict(sampling=sp.Settings()),
                dict(sampling=sp.Settings(), uniforms=_uniforms, append=True)):
        with pytest.raises(ValueError):
            _loop(synth.loop_tiny, **bad)


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 2, 64)), ("e4m3", (4, 4, 128))])
def test_a_server_step_in_a_graph(dtype, heads):
    """Logits -> tokens -> lengths -> pages and slots -> rows written -> attention, all
    captured once: sequences that draw one of the first tokens end and give their pages
    back, the others come by a row."""
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    from paper_2609_16450_gb300 import sampling as sp
    from paper_2609_16450_gb300.paged import PagedCache
    hq, hkv, D = heads
    B, d, vocab, ends = 7, 128, 1500, 60
    h = rt.Handle(E.ebd_config(
        d_model=d, vocab=vocab, n_heads_q=hq, n_heads_kv=hkv, head_dim=D, d_base=64, max_batch=B, max_window=1, max_rows=B,
        max_prefix=0, gen_len=64, g_max=5, l_min=8, l_b=32, eos_id=0, lps_enabled=1, tau=0.9, tau_psi=0.89, paged=1))
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    w = rt.DeviceWeights(w_lm=(normal(vocab, d) * 0.3).bfloat16(), w_emb=normal(vocab, 64).bfloat16())
    h.bind(w.w_emb)  # the decoding step is set up outside of captures
    i32 = dict(dtype=torch.int32, device="cuda")
    c = PagedCache(h, 9, B, 4, 16, dtype, plan="device")
    hidden, u = normal(B, d).bfloat16(), torch.zeros(B, device="cuda")
    logits, token, prob = torch.zeros((B, vocab), device="cuda"), torch.zeros(B, **i32), torch.zeros(B, device="cuda")
    draw = sp.Settings(0.8, 200, 0.95).rows(B)
    add, cu, pos = torch.zeros(B, **i32), torch.zeros(B + 1, **i32), torch.zeros(B, **i32)
    slot = torch.zeros(B, dtype=torch.int64, device="cuda")
    q, k, v = normal(B, hq, D).bfloat16(), normal(B, hkv, D).bfloat16(), normal(B, hkv, D).bfloat16()
    out = torch.zeros((B, hq, D), dtype=torch.bfloat16, device="cuda")

    def step():
        sp.lm_logits(h, hidden, w, logits)
        sp.sample(h, logits, u, token, prob, **draw)
        add.copy_(torch.where(token < ends, -c.kv_len, torch.ones_like(token)))
        c.plan(add, cu, pos, slot)
        c.write(cu, pos, k, v)
        c.attention(q, cu, c.kv_len, out, causal=True, max_new=1)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    ref = Plan(9, B, 4, 16)
    held = [[np.zeros((0, hkv, D))] * 2 for _ in range(B)]
    full = ended = 0
    for n in range(60):
        for t in (hidden, q, k, v):
            t.copy_(normal(*t.shape))
        u.copy_(torch.rand(B, generator=g, device="cuda").clamp(max=1 - 2.0 ** -24))
        out.fill_(77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        status = h.sync_status()
        tok = token.cpu().numpy()
        for b in range(B):
            sample_ref.check(logits[b].cpu().numpy(), 0.8, float(u[b]), tok[b], float(prob[b]), 200, 0.95)
        adds = [-ref.len[b] if tok[b] < ends else 1 for b in range(B)]
        rows = ref.step(adds, B)
        assert status == (E.EBD_OK if rows else E.EBD_ERR_PAGES)
        assert c.kv_len.tolist() == ref.len and c.table.tolist() == ref.table
        cus, poss, slots = rows or ([0] * (B + 1), [], [])
        assert cu.tolist() == cus and pos.tolist() == poss + [-1] * (B - len(poss))
        assert slot.tolist() == slots + [-1] * (B - len(slots))
        full += not rows
        kk, vv = ((torch.from_numpy(pr.dequantise(*pr.quantise(x.double().cpu().numpy()))) if dtype == "e4m3" else
                   x.double().cpu()).numpy() for x in (k, v))
        for b in range(B):
            if rows and adds[b] == 1:
                held[b] = [np.concatenate([a, x[cus[b]: cus[b + 1]]]) for a, x in zip(held[b], (kk, vv))]
            elif rows:
                held[b] = [x[:0] for x in held[b]]
                ended += 1
        total = cus[-1]
        assert (out[total:] == 77).all()
        if total:
            want, tol = pr.attend(q[:total].double().cpu(), [torch.from_numpy(x[0]) for x in held],
                                  [torch.from_numpy(x[1]) for x in held], [cus[b + 1] - cus[b] for b in range(B)], ref.len,
                                  hq // hkv, True, D ** -0.5)
            assert bool(((out[:total].double().cpu() - want).abs() <= tol).all())
        if not rows:  # room again: the longest ends, from outside of the graph
            b = max(range(B), key=lambda i: ref.len[i])
            gone = [-ref.len[i] if i == b else 0 for i in range(B)]
            c.plan(torch.tensor(gone, **i32))
            ref.step(gone)
            held[b] = [x[:0] for x in held[b]]
            assert h.sync_status() == E.EBD_OK
    assert full and ended
    h.close()
