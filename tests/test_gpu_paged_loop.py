"""The generation loop on a paged K/V cache: the decisions of the loop on the
dense cache, and every step's attention against its formula in 64 bits over the
rows that the pages give back."""
import numpy as np
import pytest

import synth
from tests import paged_ref as pr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _loop(sh, max_steps=None, paged=False, **opts):
    from paper_2609_16450_gb300 import loop as lp
    from paper_2609_16450_gb300 import runtime as rt
    inp = synth.make_step_inputs(sh)
    w = rt.upload_weights(inp)
    h = rt.Handle(lp.config_for_loop(sh, paged=int(paged)), w.w_emb)
    try:
        return lp.run_loop(h, sh, w, lambda s, p: synth.loop_window_inputs(sh, s, p), lambda p: synth.loop_kv(sh, p),
                           max_steps=max_steps, cache="paged" if paged else "prefix", **opts)
    finally:
        h.close()


def _f64(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).double()


@pytest.mark.parametrize("shape,steps", [("loop_tiny", None), ("loop_shape", 4)])
@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("e4m3", 64)])
def test_paged_loop(shape, steps, dtype, page):
    sh = getattr(synth, shape)
    dense = _loop(sh, steps)
    res = _loop(sh, steps, paged=True, kv_dtype=dtype, page_size=page)
    assert res.steps == dense.steps and res.commits == dense.commits
    assert np.array_equal(res.tokens, dense.tokens)
    # what the pages gave back: every row written, as it is held
    n = sh.prefix + max(r.window[1] for r in res.records)
    k, v = (_f64(x) for x in synth.loop_kv(sh, np.arange(n)))
    if dtype == "e4m3":
        k, v = (torch.from_numpy(pr.dequantise(*pr.quantise(x.numpy()))) for x in (k, v))
    got_k, got_v = _f64(res.k_cache), _f64(res.v_cache)
    assert torch.equal(got_k[:n], k) and torch.equal(got_v[:n], v)
    assert not got_k[n:].any() and not got_v[n:].any()
    k, v = k.cuda(), v.cuda()
    group = sh.n_heads_q // sh.n_heads_kv
    for r, d in zip(res.records, dense.records):
        assert r.window == d.window and np.array_equal(r.accepted, d.accepted) and np.array_equal(r.argmax, d.argmax)
        lo, hi = r.window
        q = _f64(synth.loop_window_inputs(sh, r.step, sh.prefix + np.arange(lo, hi))[1]).cuda()
        ref, tol = pr.attend(q, [k], [v], [hi - lo], [sh.prefix + hi], group, False, sh.head_dim ** -0.5)
        err = (torch.from_numpy(r.attn_out).double().cuda() - ref).abs()
        assert bool((err <= tol).all()), (r.step, float((err / tol).max()))


def test_refusals():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import loop as lp
    from paper_2609_16450_gb300 import runtime as rt
    from paper_2609_16450_gb300.paged import PagedCache
    sh = synth.loop_tiny
    w = rt.upload_weights(synth.make_step_inputs(sh))
    h = rt.Handle(lp.config_for_loop(sh), w.w_emb)
    run = lambda **o: lp.run_loop(h, sh, w, lambda s, p: synth.loop_window_inputs(sh, s, p),
                                  lambda p: synth.loop_kv(sh, p), cache="paged", **o)
    try:
        with pytest.raises(E.EbdError):  # the handle has no workspace for it
            run()
        for bad in (dict(append=True), dict(kv_dtype="fp8"), dict(page_size=48), dict(window="full", attention=False)):
            with pytest.raises(ValueError):
                run(**bad)
        c = PagedCache(h, 4, 2, 2, 16)
        i32 = dict(dtype=torch.int32, device="cuda")
        cu, pos = torch.tensor([0, 3], **i32), torch.arange(3, **i32)
        k = torch.zeros((3, c.heads, c.dim), dtype=torch.bfloat16, device="cuda")
        for call in (lambda: c.write(cu, pos, k.float(), k), lambda: c.write(cu, pos, k[:2], k),
                     lambda: c.write(cu, pos.long(), k, k), lambda: c.write(cu, pos, k[..., ::2], k[..., ::2]),
                     lambda: c.write(cu, pos, k, k, skip=torch.zeros(2, dtype=torch.uint8, device="cuda")),
                     lambda: c.read(torch.tensor([0, 1, 2, 3], **i32), pos, k, k),
                     lambda: c.attention(k, cu, cu, torch.empty_like(k)),
                     lambda: c.attention(k, cu, cu[:1], torch.empty_like(k)[:2])):
            with pytest.raises(ValueError):
                call()
    finally:
        h.close()


def test_cache_on_a_stream_of_its_own():
    """Two sequences that grow, end and give their pages to a third, on another
    stream than the current one."""
    from paper_2609_16450_gb300 import runtime as rt
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300.paged import PagedCache
    heads = (8, 2, 64)
    h = pr.handle(E, rt, heads, 3, 64)
    st = torch.cuda.Stream()
    rng = np.random.default_rng(1)
    rows = lambda n, hh: torch.from_numpy(rng.standard_normal((n, hh, 64)).astype(np.float32)).bfloat16()
    held = {b: [torch.zeros((0, 2, 64), dtype=torch.float64)] * 2 for b in range(3)}
    with torch.cuda.stream(st):
        c = PagedCache(h, 5, 3, 4, 16)
        for lens in ([20, 30, 0], [20, 30, 0], [9, None, 30], [1, 0, 1]):
            for b, n in enumerate(lens):
                if n is None:
                    c.release(b, stream=st)
                    held[b] = [x[:0] for x in held[b]]
            lens = [n or 0 for n in lens]
            need = [(len(held[b][0]) + n + 15) // 16 for b, n in enumerate(lens)]
            if sum(need) > 5:  # full: the last sequence that has rows ends
                b = max(b for b in range(3) if len(held[b][0]))
                c.release(b, stream=st)
                held[b] = [x[:0] for x in held[b]]
            new = [(rows(n, 2), rows(n, 2)) for n in lens]
            pos = np.concatenate([np.arange(len(held[b][0]), len(held[b][0]) + n) for b, n in enumerate(lens)])
            for b, n in enumerate(lens):
                held[b] = [torch.cat([a, x.double()]) for a, x in zip(held[b], new[b])]
                c.reserve(b, len(held[b][0]), stream=st)
            cu = torch.from_numpy(pr.cu_rows(lens)).cuda()
            k, v = (torch.cat([x[i] for x in new]).cuda() for i in range(2))
            c.write(cu, torch.from_numpy(pos.astype(np.int32)).cuda(), k, v, stream=st)
            q = rows(sum(lens), 8).cuda()
            out = torch.empty_like(q)
            kv = [len(held[b][0]) for b in range(3)]
            c.attention(q, cu, torch.tensor(kv, dtype=torch.int32).cuda(), out, causal=True, max_new=max(lens), stream=st)
            assert h.sync_status(st) == 0
            ref, tol = pr.attend(q.double().cpu(), [held[b][0] for b in range(3)], [held[b][1] for b in range(3)], lens,
                                 kv, 4, True, 0.125)
            assert bool(((out.double().cpu() - ref).abs() <= tol).all())
    h.close()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,rows,kv", [((28, 4, 128), [1, 1, 1], [300, 77, 2000]), ((32, 32, 128), [80, 70], [200, 900])])
def test_calls_in_a_graph(dtype, heads, rows, kv):
    """Write, attention and read captured together and replayed on new rows:
    what the calls give one by one."""
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    from paper_2609_16450_gb300.paged import PagedCache
    hq, hkv, D = heads
    n, dev = sum(rows), "cuda"
    h = pr.handle(E, rt, heads, len(rows), n)
    g = torch.Generator(device=dev).manual_seed(3)
    normal = lambda *s: torch.randn(s, generator=g, device=dev).bfloat16()
    c = PagedCache(h, 64, len(rows), 40, 64, dtype)
    for t in (c.k, c.v):
        t.copy_(torch.randint(0, 120, t.shape, generator=g, device=dev) if dtype == "e4m3" else normal(*t.shape))
    for t in (c.k_scale, c.v_scale):
        if t is not None:
            t.fill_(118)
    for b, m in enumerate(kv):
        c.reserve(b, m)
    cu = torch.from_numpy(pr.cu_rows(rows)).cuda()
    pos = torch.from_numpy(np.concatenate([np.arange(m - r, m) for r, m in zip(rows, kv)]).astype(np.int32)).cuda()
    kvl = torch.tensor(kv, dtype=torch.int32, device=dev)
    q, k, v = normal(n, hq, D), normal(n, hkv, D), normal(n, hkv, D)
    out, bk, bv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)

    def calls(stream):
        c.write(cu, pos, k, v, stream=stream)
        c.attention(q, cu, kvl, out, causal=True, max_new=max(rows), stream=stream)
        c.read(cu, pos, bk, bv, stream=stream)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        calls(st)
    for _ in range(3):
        for t in (q, k, v):
            t.copy_(normal(*t.shape))
        for _ in range(4):
            graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, bk, bv)]
        calls(torch.cuda.current_stream())
        assert h.sync_status() == 0
        for a, b in zip(got, (out, bk, bv)):
            assert torch.equal(a, b)
        if dtype == "bf16":
            assert torch.equal(bk, k) and torch.equal(bv, v)
    h.close()
