"""The paged K/V cache against its definition in 64 bits: rows written and
read back, bit for bit, and the attention over the pages."""
import math

import numpy as np
import pytest

from tests import paged_ref as pr
from tests.guards import Guarded

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HEADS = {"tiny": (4, 4, 64), "llada": (32, 32, 128), "dream": (28, 4, 128), "mqa": (8, 1, 128), "gqa64": (16, 2, 64)}


def _lib():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    return E, rt


def _bf16(rng, shape, std=1.0):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * std).bfloat16().cuda()


def _args(E, batch, rows, cu, **kw):
    a = E.ebd_paged_args()
    a.batch, a.rows, a.cu_rows = batch, rows, cu.data_ptr()
    for k, v in kw.items():
        setattr(a, k, v.data_ptr() if torch.is_tensor(v) else v)
    return a


def _special(x):
    """Rows with the values where quantising can go wrong."""
    D = x.shape[-1]
    x[0] = 0.0
    if x.shape[0] > 1:
        x[1, 0, : D // 2] = math.inf
        x[1, -1, 1] = -math.inf
    if x.shape[0] > 2:
        x[2, 0, 3] = math.nan
    if x.shape[0] > 3:
        x[3] = 2.0 ** -133  # the least bf16
        x[3, :, 5] = -3 * 2.0 ** -133
    if x.shape[0] > 4:
        x[4, :, 0] = 3.3895e38
    if x.shape[0] > 5:
        x[5, :, 2], x[5, :, 3], x[5, :, 4] = 448.0, 440.0, -424.0  # ties between codes
    if x.shape[0] > 6:
        x[6, :, 1] = 450.0
    return x


# ------------------------------------------------------------------ write and read
@pytest.mark.parametrize("heads", ["tiny", "dream", "mqa", "llada"])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,interleaved,fused", [(16, False, True), (64, True, False), (256, False, False)])
def test_write_then_read(heads, dtype, page, interleaved, fused):
    E, rt = _lib()
    hq, hkv, D = HEADS[heads]
    lens = [1, 0, 37, 64, 5, 0, 130]
    start = [0, 4, 15, 100, 63, 9, 1]
    rng = np.random.default_rng(5)
    n = sum(lens)
    total = [a + b for a, b in zip(lens, start)]
    c = pr.Cache(HEADS[heads], dtype, page, total, seed=2, interleaved=interleaved)
    h = pr.handle(E, rt, HEADS[heads], len(lens), n, paged=0)
    buf = _bf16(rng, (n, hq + 2 * hkv, D), 3.0)
    k, v = buf[:, hq: hq + hkv], buf[:, hq + hkv:]
    _special(k), _special(v)
    if not fused:
        k, v = k.contiguous(), v.contiguous()
    pos = np.concatenate([np.arange(s, s + m) for s, m in zip(start, lens)]).astype(np.int32)
    seq = np.repeat(np.arange(len(lens)), lens)
    skip = (rng.random(n) < 0.3).astype(np.uint8)
    before = [t.clone() for t in (c.k, c.v)]
    cu, posd, skipd = (torch.from_numpy(x).cuda() for x in (pr.cu_rows(lens), pos, skip))
    a = _args(E, len(lens), n, cu, row_pos=posd, k=k, v=v, skip=skipd, kv_stride=k.stride(0))
    E.check(E.ebd_paged_write(h.h, c.pages(E), a), h.h)
    out = [torch.full((n, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    a2 = _args(E, len(lens), n, cu, row_pos=posd, k=out[0], v=out[1])
    E.check(E.ebd_paged_read(h.h, c.pages(E), a2), h.h)
    assert h.sync_status() == 0
    pg, off = c.table_h[seq, pos // page], pos % page
    for rows, pool, sc, was, got in ((k, c.k, c.ks, before[0], out[0]), (v, c.v, c.vs, before[1], out[1])):
        want = was.cpu()
        if dtype == "bf16":
            want.view(torch.int16)[pg[skip == 0], :, off[skip == 0]] = rows.cpu().view(torch.int16)[skip == 0]
            assert torch.equal(pool.cpu().view(torch.int16), want.view(torch.int16))
            back = want.view(torch.int16)[pg, :, off]
            assert torch.equal(got.cpu().view(torch.int16), back)
        else:
            code, e = pr.quantise(rows.double().cpu().numpy())
            want = want.numpy()
            want[pg[skip == 0], :, off[skip == 0]] = code[skip == 0]
            np.testing.assert_array_equal(pool.cpu().numpy(), want)
            we = np.zeros(c.ks.shape, np.uint8)
            we[pg[skip == 0], :, off[skip == 0]] = e[skip == 0]
            np.testing.assert_array_equal(sc.cpu().numpy(), we)
            back = pr.dequantise(want[pg, :, off], we[pg, :, off])
            np.testing.assert_array_equal(got.double().cpu().numpy(), back)
    h.close()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_rows_without_a_page_are_left_alone(dtype):
    E, rt = _lib()
    heads = HEADS["dream"]
    hkv, D, page = heads[1], heads[2], 16
    c = pr.Cache(heads, dtype, page, [40, 40], seed=1)
    c.table_h[1, 1] = -1
    c.table_h[0, 2] = c.n_pages  # names no page
    c.table.copy_(torch.from_numpy(c.table_h))
    h = pr.handle(E, rt, heads, 2, 8, paged=0)
    pos = np.array([-1, 33, 40, 1 << 30, 20, 16, 48, 2], np.int32)
    cu = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    held = np.array([0, 0, 0, 0, 0, 0, 0, 1], bool)
    el = torch.uint8 if dtype == "e4m3" else torch.bfloat16
    k = torch.ones((8, hkv, D), dtype=torch.bfloat16, device="cuda")
    posd = torch.from_numpy(pos).cuda()
    E.check(E.ebd_paged_write(h.h, c.pages(E), _args(E, 2, 8, cu, row_pos=posd, k=k, v=k)), h.h)
    got = [torch.full((8, hkv, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    E.check(E.ebd_paged_read(h.h, c.pages(E), _args(E, 2, 8, cu, row_pos=posd, k=got[0], v=got[1])), h.h)
    assert h.sync_status() == 0
    for t in got:
        assert (t[torch.from_numpy(held).cuda()] == 1).all() and (t[torch.from_numpy(~held).cuda()] == 0).all()
    assert int((c.k.view(el) != 0).sum()) == hkv * D
    h.close()


def test_pools_past_32_bits_of_elements():
    """Pages 2^29 elements apart: the last one starts at 2.4e9 elements."""
    E, rt = _lib()
    heads, page = HEADS["mqa"], 32
    c = pr.Cache(heads, "e4m3", page, [60], seed=1, spare=4)
    c.stride = (1 << 29) + 128 * 16
    per = heads[1] * page * heads[2]
    whole = [torch.empty(c.stride * (c.n_pages - 1) + per, dtype=torch.uint8, device="cuda") for _ in range(2)]
    c.k, c.v = (torch.as_strided(w, (c.n_pages, heads[1], page, heads[2]),
                                 (c.stride, page * heads[2], heads[2], 1)) for w in whole)
    c.table_h[0, :2] = (c.n_pages - 1, c.n_pages - 2)
    c.table.copy_(torch.from_numpy(c.table_h))
    h = pr.handle(E, rt, heads, 1, 60)
    rng = np.random.default_rng(9)
    k, v, q = _bf16(rng, (60, 1, 128)), _bf16(rng, (60, 1, 128)), _bf16(rng, (60, 8, 128))
    cu = torch.tensor([0, 60], dtype=torch.int32, device="cuda")
    pos = torch.arange(60, dtype=torch.int32, device="cuda")
    E.check(E.ebd_paged_write(h.h, c.pages(E), _args(E, 1, 60, cu, row_pos=pos, k=k, v=v)), h.h)
    out = torch.zeros((60, 8, 128), dtype=torch.bfloat16, device="cuda")
    kvl = torch.tensor([60], dtype=torch.int32, device="cuda")
    E.check(E.ebd_paged_attention(h.h, c.pages(E), _args(E, 1, 60, cu, kv_len=kvl, q=q, out=out)), h.h)
    assert h.sync_status() == 0
    code, e = pr.quantise(k.double().cpu().numpy())
    np.testing.assert_array_equal(c.k[c.n_pages - 1, 0].cpu().numpy(), code[:32, 0])
    vcode, ve = pr.quantise(v.double().cpu().numpy())
    kk, vv = (torch.from_numpy(pr.dequantise(a, b)).cuda() for a, b in ((code, e), (vcode, ve)))
    ref, tol = pr.attend(q.double(), [kk], [vv], [60], [60], 8, False, 1 / math.sqrt(128))
    _close(out, ref, tol)
    h.close()


# ------------------------------------------------------------------ attention
def _close(out, ref, tol):
    err = (out.double() - ref).abs()
    assert torch.isfinite(out.float()).all()
    worst = float((err / tol).max())
    assert worst <= 1.0, f"worst error {worst} of the bound"


def _run(heads, dtype, page, lens, kv, causal, *, seed=0, interleaved=False, fused=False, scale=0.0,
         gains=(1.0, 1.0, 1.0), hint=True, edit=None, stream=None):
    E, rt = _lib()
    hq, hkv, D = HEADS[heads]
    rng = np.random.default_rng(seed)
    n = sum(lens)
    c = pr.Cache(HEADS[heads], dtype, page, kv, seed=seed, interleaved=interleaved)
    shape = (c.n_pages, hkv, page, D)
    c.fill(_bf16(rng, shape, gains[1]), _bf16(rng, shape, gains[2]))
    if edit is not None:
        edit(c)
    buf = _bf16(rng, (max(n, 1), hq + 2 * hkv, D), gains[0])
    q = buf[:, :hq]
    if not fused:
        q = q.contiguous()
    h = pr.handle(E, rt, HEADS[heads], len(lens), n)
    cu = torch.from_numpy(pr.cu_rows(lens)).cuda()
    kvl = torch.tensor(kv, dtype=torch.int32, device="cuda")
    g = Guarded(torch, max(n, 1) * hq * D, torch.bfloat16)
    a = _args(E, len(lens), n, cu, kv_len=kvl, q=q, out=g.t, q_stride=q.stride(0), causal=int(causal), scale=scale,
              max_new=max(lens) if hint else 0)
    for _ in range(2):  # twice: the workspace has to be as it was
        g.t.fill_(3.0)
        E.check(E.ebd_paged_attention(h.h, c.pages(E), a, rt.stream_handle(stream)), h.h)
    assert h.sync_status(stream) == 0
    assert g.intact()
    h.close()
    out = g.t.view(-1, hq, D)[:n]
    return c, q[:n], out


def _check(heads, dtype, page, lens, kv, causal, **kw):
    c, q, out = _run(heads, dtype, page, lens, kv, causal, **kw)
    hq, hkv, D = HEADS[heads]
    scale = kw.get("scale") or 1 / math.sqrt(D)
    k, v = ([c.rows_of(i, b, m) for b, m in enumerate(kv)] for i in (0, 1))
    ref, tol = pr.attend(q.double(), k, v, lens, kv, hq // hkv, causal, scale)
    _close(out, ref, tol)
    return out


LENS = {  # new rows, cached positions
    "one_token": ([1], [1]),
    "tokens": ([1, 1, 1, 1, 1], [1, 17, 64, 65, 700]),
    "window": ([32], [160]),
    "ragged": ([5, 0, 33, 64, 1, 16], [5, 0, 100, 64, 513, 255]),
    "nothing_cached": ([4, 2, 3], [0, 130, 0]),
    "chunk": ([200, 3], [331, 3]),
}


@pytest.mark.parametrize("heads", sorted(HEADS))
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens", sorted(LENS))
@pytest.mark.parametrize("causal", [False, True])
def test_attention(heads, dtype, lens, causal):
    n, kv = LENS[lens]
    page = {"tiny": 16, "llada": 64, "dream": 32, "mqa": 128, "gqa64": 256}[heads]
    _check(heads, dtype, page, n, kv, causal, seed=7, fused=heads == "dream", interleaved=heads == "gqa64",
           hint=lens != "ragged")


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attention_pages(dtype, page):
    _check("dream", dtype, page, [9, 2], [page * 3 + 1, page - 1], False, seed=page)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n", [("mqa", 1), ("dream", 4), ("llada", 40), ("tiny", 64), ("dream", 64), ("mqa", 100)])
def test_attention_split_over_a_long_cache(dtype, heads, n):
    """Few rows over 20011 positions: tiles in many parts."""
    _check(heads, dtype, 64, [n], [20011], False, seed=n)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,n", [("llada", 65), ("llada", 128), ("llada", 129), ("dream", 18), ("dream", 19),
                                     ("dream", 37), ("mqa", 33)])
@pytest.mark.parametrize("kv", [140, 128, 256, 129, 1500])
def test_attention_tiles(dtype, causal, heads, n, kv):
    """One tile of up to 128 packed rows, two, three; one step of 128 keys and more."""
    _check(heads, dtype, 128, [n], [kv], causal, seed=n + kv)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_attention_causal_rows_that_see_nothing(dtype):
    """More new rows than cached positions: the first ones see none."""
    for heads in ("dream", "tiny"):
        out = _check(heads, dtype, 16, [20, 3], [7, 3], True, seed=3)
        assert (out[:13] == 0).all() and (out[13:20] != 0).any()
    out = _check("llada", dtype, 16, [300], [100], True, seed=3)
    assert (out[:200] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n", [("dream", 3), ("llada", 64), ("dream", 150)])
def test_what_pages_hold_past_the_end_has_no_part(dtype, heads, n):
    def garbage(c):
        for b, m in enumerate([333, 64]):
            for i in range(c.max_pages):
                pg = c.table_h[b, i]
                lo = max(0, min(c.page, m - i * c.page))
                if pg < 0 or lo == c.page:
                    continue
                for pool in (c.k, c.v):
                    pool[pg, :, lo:] = 0x7F if c.dtype == "e4m3" else math.nan
                    if c.dtype == "bf16":
                        pool[pg, :, lo::2] = math.inf
                if c.ks is not None:
                    c.ks[pg, :, lo:] = 255
                    c.vs[pg, :, lo:] = 255
        held = set(c.table_h.ravel().tolist())
        for pg in range(c.n_pages):
            if pg not in held:
                c.k[pg] = 0x7F if c.dtype == "e4m3" else math.nan
                c.v[pg] = 0x7F if c.dtype == "e4m3" else math.nan

    for causal in (False, True):
        c, q, out = _run(heads, dtype, 32, [n, 2], [333, 64], causal, seed=4, edit=garbage)
        hq, hkv, D = HEADS[heads]
        k, v = ([c.rows_of(i, b, m) for b, m in enumerate([333, 64])] for i in (0, 1))
        ref, tol = pr.attend(q.double(), k, v, [n, 2], [333, 64], hq // hkv, causal, 1 / math.sqrt(D))
        _close(out, ref, tol)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n,kv", [("dream", 30, 95), ("llada", 70, 300), ("mqa", 200, 210)])
@pytest.mark.parametrize("what", ["nan", "inf", "-inf", "nan_key"])
def test_causal_rows_before_a_value_that_is_not_finite(dtype, heads, n, kv, what):
    """Position j of the chunk holds one: the rows before it do not see it, the
    others have it in that element (a key: in the whole row)."""
    if dtype == "e4m3" and "inf" in what:
        pytest.skip("8 bits hold no infinities")
    j, d, hk = kv - n + n // 2, 37, 0
    whole = what == "nan_key" or dtype == "e4m3"  # the row's result as a whole, or element d
    was = {}

    def edit(c):
        pool, sc = (c.k, c.ks) if what == "nan_key" else (c.v, c.vs)
        at = (int(c.table_h[0, j // c.page]), hk, j % c.page)
        was.update(pool=pool, sc=sc, at=at, x=pool[at].clone(), e=sc[at].clone() if sc is not None else None)
        if dtype == "e4m3":
            pool[at], sc[at] = 0x7F, 255
        else:
            pool[at][d] = float(what.split("_")[0])

    c, q, out = _run(heads, dtype, 64, [n], [kv], True, seed=6, edit=edit)
    hq, hkv, D = HEADS[heads]
    g = hq // hkv
    see = torch.arange(n, device="cuda") >= j - (kv - n)
    mine = torch.zeros_like(out, dtype=torch.bool)
    mine[:, hk * g: (hk + 1) * g, slice(None) if whole else d] = see.view(-1, 1, 1) if whole else see[:, None]
    bad = out[mine].float()
    assert {"n": torch.isnan(bad), "i": bad == math.inf, "-": bad == -math.inf}[what[0]].all()
    # everything else as if the row were what it was
    was["pool"][was["at"]] = was["x"]
    if was["sc"] is not None:
        was["sc"][was["at"]] = was["e"]
    k, v = ([c.rows_of(i, 0, kv)] for i in (0, 1))
    ref, tol = pr.attend(q.double(), k, v, [n], [kv], g, True, 1 / math.sqrt(D))
    _close(torch.where(mine, ref.bfloat16(), out), ref, tol)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("gains", [(40.0, 1.0, 1.0), (1.0, 100.0, 1e-6), (1e-3, 1.0, 3e6), (0.0, 1.0, 1.0)])
@pytest.mark.parametrize("heads,n", [("dream", 2), ("llada", 33), ("mqa", 90)])
def test_attention_magnitudes(dtype, gains, heads, n):
    """Scores of some hundred and of none, values small and past 2^9 * 448."""
    _check(heads, dtype, 32, [n], [500], False, seed=8, gains=gains,
           scale=0.01 if gains[1] > 10 else 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_attention_keys_that_rise(dtype):
    """Scores that grow along the cache: the running maximum moves all the time."""
    def ramp(c):
        rng = np.random.default_rng(1)
        k = _bf16(rng, (c.n_pages, c.hkv, c.page, c.D))
        for i in range(c.max_pages):
            k[int(c.table_h[0, i])] *= 0.2 + 0.2 * i
        c.fill(k, _bf16(rng, k.shape))

    _check("dream", dtype, 16, [5], [777], False, seed=2, edit=ramp, gains=(2.0, 1.0, 1.0))
    _check("mqa", dtype, 16, [90], [777], False, seed=2, edit=ramp, gains=(2.0, 1.0, 1.0))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n", [("dream", 3), ("tiny", 20), ("gqa64", 5), ("llada", 40), ("mqa", 100)])
@pytest.mark.parametrize("what", ["wide", "zero"])
def test_attention_values_of_wide_range(dtype, heads, n, what):
    """Values from 2^-30 to 2^30, or none, position by position, and sharp scores:
    a row's result is that of the keys it looks at, whatever the others hold."""
    def wide(c):
        rng = np.random.default_rng(12)
        k, v = (_bf16(rng, (c.n_pages, c.hkv, c.page, c.D)) for _ in range(2))
        by = (c.n_pages, c.hkv, c.page, 1)
        f = np.exp2(rng.integers(-30, 31, by)) if what == "wide" else (rng.random(by) < 0.5) * 1.0
        c.fill(k, (v * torch.from_numpy(f.astype(np.float32)).cuda()).bfloat16())

    _check(heads, dtype, 64, [n], [700], False, seed=11, gains=(6.0, 1.0, 1.0), edit=wide)


def test_attention_on_another_stream():
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _check("dream", "e4m3", 64, [3, 40], [100, 900], True, seed=5, stream=s)


@pytest.mark.parametrize("batch", [300, 1111])
def test_attention_many_sequences(batch):
    rng = np.random.default_rng(batch)
    n = rng.integers(0, 4, batch).tolist()
    kv = [int(m + rng.integers(0, 60)) for m in n]
    _check("gqa64", "bf16", 16, n, kv, True, seed=1)


def test_attention_results_do_not_depend_on_the_run():
    outs = [_run("dream", "e4m3", 64, [7, 30], [9000, 300], False, seed=3)[2].clone() for _ in range(3)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ------------------------------------------------------------------ refusals
def test_refusals():
    E, rt = _lib()
    heads = HEADS["dream"]
    c = pr.Cache(heads, "e4m3", 64, [100])
    h = pr.handle(E, rt, heads, 2, 16)
    t = torch.zeros(16 * 28 * 128 + 8, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, 4], dtype=torch.int32, device="cuda")

    def args(**kw):
        a = _args(E, 1, 4, cu, row_pos=cu, kv_len=cu, q=t, k=t, v=t, out=t)
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    def pages(**kw):
        p = c.pages(E)
        for k, v in kw.items():
            setattr(p, k, v)
        return p

    every = (E.ebd_paged_write, E.ebd_paged_read, E.ebd_paged_attention)
    bad_pages = [dict(dtype=2), dict(dtype=-1), dict(page_size=8), dict(page_size=48), dict(page_size=512),
                 dict(n_pages=0), dict(max_pages=0), dict(k=None), dict(v=None), dict(page_table=None),
                 dict(k=c.k.data_ptr() + 8), dict(k_scale=None), dict(v_scale=c.vs.data_ptr() + 1),
                 dict(page_stride=64), dict(page_stride=4 * 64 * 128 + 8)]
    for kw in bad_pages:
        for fn in every:
            assert fn(h.h, pages(**kw), args()) == E.EBD_ERR_INVALID_ARG, kw
    for kw in (dict(batch=3), dict(batch=-1), dict(rows=17), dict(rows=-1), dict(cu_rows=None), dict(batch=0)):
        for fn in every:
            assert fn(h.h, pages(), args(**kw)) == E.EBD_ERR_INVALID_ARG, kw
    for kw in (dict(row_pos=None), dict(k=None), dict(v=t.data_ptr() + 2), dict(kv_stride=128), dict(kv_stride=516)):
        for fn in every[:2]:
            assert fn(h.h, pages(), args(**kw)) == E.EBD_ERR_INVALID_ARG, kw
    for kw in (dict(kv_len=None), dict(q=None), dict(out=None), dict(q=t.data_ptr() + 2), dict(out=t.data_ptr() + 4),
               dict(q_stride=1), dict(q_stride=28 * 128 + 4), dict(causal=2), dict(max_new=-1),
               dict(scale=math.nan), dict(scale=math.inf), dict(scale=-1.0)):
        assert E.ebd_paged_attention(h.h, pages(), args(**kw)) == E.EBD_ERR_INVALID_ARG, kw
        assert E.ebd_last_error(h.h)
    for fn in every:
        assert fn(None, pages(), args()) == E.EBD_ERR_INVALID_ARG
        assert fn(h.h, pages(), args(rows=0, batch=0)) == E.EBD_OK
    h0 = pr.handle(E, rt, heads, 1, 4, paged=0)
    assert E.ebd_paged_attention(h0.h, pages(), args()) == E.EBD_ERR_STATE
    s, hh = E.ebd_create(E.ebd_config(
        d_model=64, vocab=64, n_heads_q=4, n_heads_kv=4, head_dim=64, d_base=64, max_batch=1, max_window=1,
        max_rows=1, gen_len=1, tau=0.9, tau_psi=0.9, paged=2))
    assert s == E.EBD_ERR_UNSUPPORTED
    h0.close()
    assert h.sync_status() == 0
    h.close()


def test_a_position_without_a_page_is_reported():
    E, rt = _lib()
    heads = HEADS["tiny"]
    c = pr.Cache(heads, "bf16", 16, [64])
    c.table_h[0, 2] = -1
    c.table.copy_(torch.from_numpy(c.table_h))
    h = pr.handle(E, rt, heads, 1, 4)
    q = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    g = Guarded(torch, q.numel(), torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    kvl = torch.tensor([64], dtype=torch.int32, device="cuda")
    a = _args(E, 1, 4, cu, kv_len=kvl, q=q, out=g.t)
    E.check(E.ebd_paged_attention(h.h, c.pages(E), a), h.h)
    assert h.sync_status() == E.EBD_ERR_BOUNDS and g.intact()
    kvl.fill_(32)
    E.check(E.ebd_paged_attention(h.h, c.pages(E), a), h.h)
    assert h.sync_status() == 0
    kvl.fill_(-5)  # no positions
    E.check(E.ebd_paged_attention(h.h, c.pages(E), a), h.h)
    assert h.sync_status() == 0 and (g.t == 0).all()
    h.close()
