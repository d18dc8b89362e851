"""The paged attention where its kernels' waits, references and records could go
wrong: values that are not finite in many places, scores past what 32 bits
resolve, values of very unequal size, calls that give up."""
import math

import numpy as np
import pytest

from tests import paged_ref as pr
from tests.test_gpu_paged import HEADS, _args, _close, _lib, _run

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _reference(c, q, heads, lens, kv, causal, scale=0.0):
    hq, hkv, D = HEADS[heads]
    k, v = ([c.rows_of(i, b, m) for b, m in enumerate(kv)] for i in (0, 1))
    return pr.attend(q.double(), k, v, lens, kv, hq // hkv, causal, scale or 1 / math.sqrt(D))


def _attend(c, heads, q, lens, kv, causal=False):
    """The attention of rows q over a cache that is there."""
    E, rt = _lib()
    h = pr.handle(E, rt, HEADS[heads], len(lens), sum(lens))
    cu = torch.from_numpy(pr.cu_rows(lens)).cuda()
    kvl = torch.tensor(kv, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    a = _args(E, len(lens), sum(lens), cu, kv_len=kvl, q=q, out=out, causal=int(causal), max_new=max(lens))
    E.check(E.ebd_paged_attention(h.h, c.pages(E), a, rt.stream_handle(None)), h.h)
    assert h.sync_status() == 0
    h.close()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n,kv", [("llada", 100, 128), ("llada", 150, 256), ("mqa", 9, 128), ("dream", 37, 140)])
def test_causal_nan_values_all_over_many_short_tiles(dtype, heads, n, kv):
    """Tiles of one and two steps, several per SM, each with value rows that are
    NaN among the keys that only some of its rows see, in the key ranges of
    several warps: the rows before them are as without them."""
    hq, hkv, D = HEADS[heads]
    page, batch = 64, min(4096 // n, max(28, 500 // hkv))
    lens, kvs = [n] * batch, [kv] * batch
    rng = np.random.default_rng(17)
    # (sequence, head, key, element): up to 5 a head
    b, h = (x.ravel() for x in np.meshgrid(np.arange(batch), np.arange(hkv), indexing="ij"))
    b, h = np.repeat(b, 5), np.repeat(h, 5)
    keep = rng.random(b.size) < 0.6
    b, h = b[keep], h[keep]
    key = rng.integers(kv - n, kv, b.size)
    d = rng.integers(0, D, b.size)
    was = {}

    def edit(c):
        at = [torch.from_numpy(x.astype(np.int64)).cuda() for x in (c.table_h[b, key // page], h, key % page)]
        was.update(at=at, v=c.v.clone(), vs=None if c.vs is None else c.vs.clone())
        if dtype == "e4m3":
            c.v[tuple(at)] = 0x7F
            c.vs[tuple(at)] = 255
        else:
            c.v[tuple(at) + (torch.from_numpy(d).cuda(),)] = math.nan

    c, q, out = _run(heads, dtype, page, lens, kvs, True, seed=21, edit=edit)
    # first key of each (sequence, head, element) that is NaN
    first = np.full((batch, hkv, D), kv + 1)
    if dtype == "e4m3":
        np.minimum.at(first, (b, h), key[:, None])
    else:
        np.minimum.at(first, (b, h, d), key)
    limit = kv - n + np.arange(n) + 1
    bad = limit[None, :, None, None] > first[:, None]                       # [batch][n][hkv][D]
    bad = torch.from_numpy(np.repeat(bad, hq // hkv, axis=2).reshape(batch * n, hq, D)).cuda()
    assert torch.isnan(out[bad].float()).all()
    c.v.copy_(was["v"])
    if c.vs is not None:
        c.vs.copy_(was["vs"])
    ref, tol = _reference(c, q, heads, lens, kvs, True)
    _close(torch.where(bad, ref.bfloat16(), out), ref, tol)


# packed rows on either kernel, over caches that are whole and cut into parts
HUGE = [("llada", 70, 500), ("mqa", 20, 3000), ("dream", 40, 500), ("llada", 200, 3000),
        ("dream", 2, 500), ("llada", 20, 3000), ("tiny", 40, 700), ("gqa64", 5, 500)]


def _bound(ref, v, lens, group):
    """What rounding a probability and the result to bf16 may change (as in paged_ref.attend)."""
    mag = torch.cat([vv.abs().mean(0).repeat_interleave(group, 0).expand(n, -1, -1) for n, vv in zip(lens, v)])
    return 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12) * mag + 1e-30


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n,kv", HUGE)
@pytest.mark.parametrize("size", [1e4, 1e5, 1e9, 1e17])
def test_equal_scores_of_any_size_share_alike(dtype, heads, n, kv, size):
    """All keys of a head alike, with scores past what 32 bits resolve: every
    row's result is its values' mean."""
    hq, hkv, D = HEADS[heads]

    def alike(c):
        rng = np.random.default_rng(3)
        k = torch.from_numpy(rng.standard_normal((1, hkv, 1, D)).astype(np.float32) * np.float32(size)).cuda()
        v = torch.from_numpy(rng.standard_normal((c.n_pages, hkv, c.page, D)).astype(np.float32)).cuda()
        c.fill(k.expand(c.n_pages, hkv, c.page, D).bfloat16().contiguous(), v.bfloat16())

    c, q, out = _run(heads, dtype, 64, [n], [kv], False, seed=31, gains=(size, 1.0, 1.0), edit=alike)
    v = [c.rows_of(1, 0, kv)]
    ref = v[0].mean(0).repeat_interleave(hq // hkv, 0).expand(n, -1, -1)
    _close(out, ref, _bound(ref, v, [n], hq // hkv))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n,kv", HUGE)
@pytest.mark.parametrize("size", [1e4, 1e5, 1e9, 1e17])
def test_scores_of_any_size_pick_the_largest(dtype, heads, n, kv, size):
    """Scores past what 32 bits resolve: rows whose largest score stands out by
    more than their rounding have that key's values, all have a mean of values."""
    hq, hkv, D = HEADS[heads]
    c, q, out = _run(heads, dtype, 64, [n], [kv], False, seed=32, gains=(size, size, 1.0))
    k, v = (c.rows_of(i, 0, kv) for i in (0, 1))
    o = out.double()
    assert torch.isfinite(o).all()
    for h in range(hq):
        kk, vv = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        s = q[:, h].double() @ kk.T / math.sqrt(D)
        assert (o[:, h] <= vv.amax(0) + 2.0 ** -7 * vv.abs().amax(0)).all()
        assert (o[:, h] >= vv.amin(0) - 2.0 ** -7 * vv.abs().amax(0)).all()
        top = s.topk(2, -1)
        # rounding of a score: 2^-17 of sum |q||k| scale (paged_ref.attend), twice
        err = 2.0 ** -16 * (q[:, h].double().abs() @ kk.abs().T / math.sqrt(D)).amax(-1)
        clear = top.values[:, 0] - top.values[:, 1] > err + 40.0
        assert clear.any()
        want = vv[top.indices[clear, 0]]
        # P and its sum: one probability, rounded or not
        assert ((o[clear, h] - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -30).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n,kv", [("llada", 70, 128), ("llada", 70, 300), ("llada", 200, 300), ("mqa", 20, 3000),
                                        ("dream", 40, 128)])
@pytest.mark.parametrize("gap", [26.0, 31.0])
def test_second_halves_of_steps_far_above_the_first(dtype, heads, n, kv, gap):
    """Of every 128 keys the last 64 score some 2^gap above the others, whose
    values are as much larger: what a row has of a step's first half counts,
    although its reference moves past 2^24 of it in the second."""
    hq, hkv, D = HEADS[heads]
    rng = np.random.default_rng(5)
    # a direction per K/V head that q and the second halves' keys share
    u = rng.standard_normal((hkv, D)).astype(np.float32)
    u /= np.linalg.norm(u, axis=-1, keepdims=True)
    want = gap * math.log(2) * math.sqrt(D)  # q . k

    def edit(c):
        k = rng.standard_normal((c.n_pages, hkv, c.page, D)).astype(np.float32) * 0.1
        v = rng.standard_normal(k.shape).astype(np.float32)
        for i in range(c.max_pages):
            pg = int(c.table_h[0, i])
            if i % 2:
                k[pg] += 0.1 * want * u[:, None]
            else:
                v[pg] *= 2.0 ** gap
        c.fill(torch.from_numpy(k).cuda().bfloat16(), torch.from_numpy(v).cuda().bfloat16())

    c = pr.Cache(HEADS[heads], dtype, 64, [kv], seed=4)
    edit(c)
    q = np.repeat(10.0 * u, hq // hkv, axis=0)[None] + 0.3 * rng.standard_normal((n, hq, D))
    q = torch.from_numpy(q.astype(np.float32)).cuda().bfloat16()
    out = _attend(c, heads, q, [n], [kv])
    ref, tol = _reference(c, q, heads, [n], [kv], False)
    _close(out, ref, tol)
    # both halves of the steps count
    p = torch.softmax(q[:, 0].double() @ c.rows_of(0, 0, kv)[:, 0].T / math.sqrt(D), -1)
    lo = p[:, torch.arange(kv, device="cuda") % 128 < 64].sum(-1) * 2.0 ** gap
    assert 2.0 ** -4 < float(lo.median()) < 2.0 ** 4


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n", [("dream", 2), ("llada", 30), ("mqa", 40), ("dream", 40)])
def test_a_call_that_gives_up_writes_nothing_of_an_earlier_one(dtype, heads, n):
    """A call of two sequences over long caches, whose tiles are put together
    from parts; then one of a single row or tile that gives up: it reports so, and
    no row past its own is written.  The next call is as ever."""
    E, rt = _lib()
    hq, hkv, D = HEADS[heads]
    kv = [4000, 9000]
    rng = np.random.default_rng(8)
    c = pr.Cache(HEADS[heads], dtype, 64, kv, seed=8)
    x = [torch.from_numpy(rng.standard_normal((c.n_pages, hkv, 64, D)).astype(np.float32)).cuda().bfloat16() for _ in range(2)]
    c.fill(*x)
    q = torch.from_numpy(rng.standard_normal((2 * n, hq, D)).astype(np.float32)).cuda().bfloat16()
    cfg = E.ebd_config(
        d_model=64, vocab=64, n_heads_q=hq, n_heads_kv=hkv, head_dim=D, d_base=64, max_batch=2, max_window=1,
        max_rows=2 * n, max_prefix=0, gen_len=1, g_max=5, l_min=8, l_b=32, eos_id=63, lps_enabled=1, tau=0.9,
        tau_psi=0.89, debug_flags=E.EBD_DEBUG_PAGED_GIVE_UP, paged=1)
    h = rt.Handle(cfg)
    out = torch.full((2 * n, hq, D), 3.0, dtype=torch.bfloat16, device="cuda")

    def call(lens):
        cu = torch.from_numpy(pr.cu_rows(lens)).cuda()
        kvl = torch.tensor(kv[: len(lens)], dtype=torch.int32, device="cuda")
        a = _args(E, len(lens), sum(lens), cu, kv_len=kvl, q=q, out=out, max_new=max(lens))
        E.check(E.ebd_paged_attention(h.h, c.pages(E), a, rt.stream_handle(None)), h.h)
        return h.sync_status()

    assert call([n, n]) == 0
    ref, tol = _reference(c, q, heads, [n, n], kv, False)
    _close(out, ref, tol)
    out.fill_(5.0)
    assert call([1]) == E.EBD_ERR_TIMEOUT
    assert (out[1:] == 5.0).all()
    assert call([n, n]) == 0
    _close(out, ref, tol)
    h.close()


def _along(rng, heads, c, kv, score, value):
    """Fills a cache so that key j scores score[j] log2 units above key noise and
    its values are about value[j]; returns rows of q."""
    hq, hkv, D = HEADS[heads]
    u = rng.standard_normal((hkv, D)).astype(np.float32)
    u /= np.linalg.norm(u, axis=-1, keepdims=True)
    k = 0.1 * rng.standard_normal((c.n_pages, hkv, c.page, D)).astype(np.float32)
    v = rng.standard_normal(k.shape).astype(np.float32)
    for j in range(kv):
        at = (int(c.table_h[0, j // c.page]), slice(None), j % c.page)
        k[at] += 0.1 * math.log(2) * math.sqrt(D) * score[j] * u
        v[at] *= np.float32(value[j])
    c.fill(torch.from_numpy(k).cuda().bfloat16(), torch.from_numpy(v).cuda().bfloat16())
    q = np.repeat(10.0 * u, hq // hkv, axis=0)[None] + 0.1 * rng.standard_normal((8, hq, D))
    return torch.from_numpy(q.astype(np.float32)).cuda().bfloat16()


FEW = ["dream", "tiny", "gqa64", "llada"]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads", FEW)
@pytest.mark.parametrize("steps", [(-60, -20, 20, 60), (-40, -25, -10, 5, 20, 35), (-84, -42, 0, 42, 84)])
def test_values_that_grow_behind_the_keys_that_count(dtype, heads, steps):
    """Values larger chunk by chunk, all of a row's weight on the first chunk: the
    row has that chunk's values."""
    kv = 64 * len(steps)
    rng = np.random.default_rng(13)
    c = pr.Cache(HEADS[heads], dtype, 64, [kv], seed=3)
    score = np.where(np.arange(kv) < 64, 400.0, 0.0)
    q = _along(rng, heads, c, kv, score, np.repeat(np.exp2(np.array(steps, float)), 64))
    out = _attend(c, heads, q, [8], [kv])
    ref, tol = _reference(c, q, heads, [8], [kv], False)
    assert float(ref.abs().max()) < 2.0 ** (steps[0] + 4)
    _close(out, ref, tol)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads", FEW)
@pytest.mark.parametrize("gap", [60.0, 100.0, 126.0, 140.0, 300.0, 2000.0])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -30])
def test_a_key_far_above_the_others_whose_values_are_small(dtype, heads, gap, small):
    """Values past 2^9, but small or zero ones at some key of the second chunk that
    scores far above all others: its values are the row's."""
    kv = 200
    rng = np.random.default_rng(14)
    c = pr.Cache(HEADS[heads], dtype, 64, [kv], seed=3)
    key = np.arange(kv) == 101
    q = _along(rng, heads, c, kv, np.where(key, gap, 0.0), np.where(key, small, 2.0 ** 12))
    out = _attend(c, heads, q, [8], [kv])
    ref, tol = _reference(c, q, heads, [8], [kv], False)
    _close(out, ref, tol)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,n,kv,gain", [("llada", 70, 500, 12.0), ("mqa", 60, 3000, 60.0), ("dream", 40, 900, 12.0),
                                             ("llada", 200, 1500, 12.0)])
def test_rows_that_look_at_one_key_have_its_values(dtype, heads, n, kv, gain):
    """Sharp rows over caches that take tcgen05: a row whose other keys weigh less
    than 2^-20 together has its key's values, as they are in the cache."""
    hq, hkv, D = HEADS[heads]
    c, q, out = _run(heads, dtype, 64, [n], [kv], False, seed=33, gains=(gain, 1.0, 1.0))
    k, v = (c.rows_of(i, 0, kv) for i in (0, 1))
    seen = 0
    for h in range(hq):
        kk, vv = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        p = torch.softmax(q[:, h].double() @ kk.T / math.sqrt(D), -1)
        top = p.max(-1)
        one = 1 - top.values < 2.0 ** -20
        # others' weight times what they hold, and 32-bit sums, far below bf16's half step
        want = vv[top.indices[one]]
        far = (1 - top.values[one])[:, None] * vv.abs().amax() > 2.0 ** -12 * want.abs()
        got = out[one, h].double()
        assert (far | (got == want)).all()
        seen += int((~far).sum())
    assert seen > 1000


def test_page_tables_wider_than_positions_count_are_refused():
    """kv_len is cut to the page table; past 2^31 - 256 positions the last steps'
    ends would not fit 32 bits."""
    E, rt = _lib()
    c = pr.Cache(HEADS["tiny"], "bf16", 256, [100])
    h = pr.handle(E, rt, HEADS["tiny"], 1, 1)
    cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    a = _args(E, 1, 1, cu, kv_len=cu[1:], q=q, out=torch.empty_like(q))
    for pages in (1 << 23, (1 << 31) - 1):
        p = c.pages(E)
        p.max_pages = pages
        assert E.ebd_paged_attention(h.h, p, a, rt.stream_handle(None)) == E.EBD_ERR_UNSUPPORTED
    assert h.sync_status() == 0
    h.close()
