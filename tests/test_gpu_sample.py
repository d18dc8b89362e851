"""ebd_sample against the definition in 64 bits: vocabularies, types, strides,
filters, ties, masks, and rows that are refused."""
import numpy as np
import pytest

from tests import sample_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F32 = dict(dtype=torch.float32, device="cuda")


def _lib():
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    return E, rt


def handle(vocab, rows=512):
    E, rt = _lib()
    return rt.Handle(E.ebd_config(
        d_model=64, vocab=vocab, n_heads_q=4, n_heads_kv=4, head_dim=64, d_base=64, max_batch=rows, max_window=64,
        max_rows=rows, max_prefix=0, gen_len=64, g_max=5, l_min=8, l_b=32, eos_id=0, lps_enabled=1, tau=0.9, tau_psi=0.89,
        paged=1))


def _dev(x, dtype):
    return None if x is None else torch.as_tensor(np.asarray(x), dtype=dtype).cuda()


def sample(h, logits, u, T=None, k=None, p=None, q=None, stream=None):
    """token, prob, status of one call."""
    E, rt = _lib()
    rows = logits.shape[0]
    keep = [_dev(u, torch.float32), _dev(T, torch.float32), _dev(k, torch.int32), _dev(p, torch.float32),
            _dev(q, torch.float32)]
    token = torch.full((rows + 2,), 77, dtype=torch.int32, device="cuda")
    prob = torch.full((rows + 2,), 77.0, **F32)
    a = E.ebd_sample_args()
    a.rows, a.dtype = rows, {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[logits.dtype]
    a.logits, a.stride = logits.data_ptr(), logits.stride(0)
    a.u, a.temperature, a.top_k, a.top_p, a.min_p = (rt.ptr(t) for t in keep)
    a.token, a.prob = token.data_ptr() + 4, prob.data_ptr() + 4
    E.check(E.ebd_sample(h.h, a, rt.stream_handle(stream)), h.h)
    status = h.sync_status(stream)
    for t in (token, prob):
        assert t[0] == 77 and t[-1] == 77
    return token[1:-1].cpu().numpy(), prob[1:-1].cpu().numpy(), status


def make(rows, vocab, dtype="f32", pad=0, offset=0, seed=0, banned=0.05):
    """Rows of unequal sharpness, some tokens banned, in a wider buffer."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, vocab)) * np.exp(g.uniform(np.log(0.3), np.log(8), (rows, 1)))
    mask = g.uniform(size=(rows, vocab)) < banned * (g.uniform(size=(rows, 1)) < 0.5)
    mask[np.arange(rows), g.integers(0, vocab, rows)] = False
    x[mask] = -np.inf
    buf = torch.full((rows * (vocab + pad) + offset + 8,), float("nan"), dtype=DTYPES[dtype], device="cuda")
    t = buf[offset: offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    t.copy_(torch.from_numpy(x))
    return t, g


def params(g, rows, vocab, filters):
    T = np.exp(g.uniform(np.log(0.2), np.log(2), rows)).astype(np.float32)
    k = p = q = None
    if "k" in filters:
        k = np.exp(g.uniform(0, np.log(vocab), rows)).astype(np.int32)
        k[::5] = 0
    if "p" in filters:
        p = g.uniform(0, 1.1, rows).astype(np.float32)
    if "q" in filters:
        q = np.exp(g.uniform(np.log(1e-4), 0, rows)).astype(np.float32)
        q[::4] = 0
    if "0" in filters:
        T[::2] = 0
    return T, k, p, q, g.uniform(0, 1, rows).astype(np.float32) * np.float32(1 - 2 ** -24)


def verify(logits, T, k, p, q, u, token, prob):
    l = logits.float().cpu().numpy()
    for r in range(len(token)):
        ref.check(l[r], 1.0 if T is None else T[r], u[r], token[r], prob[r], 0 if k is None else k[r],
                  1.0 if p is None else p[r], 0.0 if q is None else q[r])


@pytest.mark.parametrize("filters", ["", "k", "p", "q", "kp", "kpq", "kpq0"])
@pytest.mark.parametrize("vocab,rows", [(2, 5), (31, 40), (500, 30), (4096, 24), (57381, 16), (152064, 9), (700001, 4)])
def test_filters(vocab, rows, filters):
    h = handle(vocab)
    logits, g = make(rows, vocab, seed=vocab + len(filters))
    T, k, p, q, u = params(g, rows, vocab, filters)
    token, prob, status = sample(h, logits, u, T, k, p, q)
    assert status == 0
    verify(logits, T, k, p, q, u, token, prob)
    h.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (3, 5), (8, 1), (57, 7)])
def test_types_and_strides(dtype, pad, offset):
    """16-bit logits tie often: kept shares end within equal ones."""
    for vocab in (517, 33001):
        h = handle(vocab)
        logits, g = make(12, vocab, dtype, pad, offset, seed=pad * 10 + offset)
        T, k, p, q, u = params(g, 12, vocab, "kpq")
        token, prob, status = sample(h, logits, u, T, k, p, q)
        assert status == 0
        verify(logits, T, k, p, q, u, token, prob)
        h.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,rows", [(517, 100), (33001, 100), (33001, 200), (130003, 80)])
def test_many_rows(dtype, vocab, rows):
    """More rows than run at once: another kernel, on one or two CTAs a row."""
    h = handle(vocab)
    for filters in ("", "kp", "pq"):
        logits, g = make(rows, vocab, dtype, 1, 3, seed=vocab + rows)
        T, k, p, q, u = params(g, rows, vocab, filters + "0" if filters == "kp" else filters)
        token, prob, status = sample(h, logits, u, T, k, p, q)
        assert status == 0
        verify(logits, T, k, p, q, u, token, prob)
    h.close()


@pytest.mark.parametrize("vocab", [6, 4096, 100003])
def test_equal_logits(vocab):
    """All equal, and in groups of equals: kept by index."""
    h = handle(vocab)
    g = np.random.default_rng(3)
    rows = 24
    x = np.zeros((rows, vocab), np.float32)
    x[8:] = np.floor(g.uniform(0, 3, (rows - 8, vocab)))
    x[16:, ::2] *= -0.0  # -0 and 0 are equal
    T = np.full(rows, 0.7, np.float32)
    k = g.integers(0, vocab, rows).astype(np.int32)
    p = g.uniform(0, 1, rows).astype(np.float32)
    p[::3], k[1::3] = 1.0, 0
    u = g.uniform(0, 1, rows).astype(np.float32) * np.float32(1 - 2 ** -24)
    logits = torch.from_numpy(x).cuda()
    token, prob, status = sample(h, logits, u, T, k, p, None)
    assert status == 0
    verify(logits, T, k, p, None, u, token, prob)
    h.close()


def test_borders_at_zero():
    """-0 and 0 are equal, and between the smallest numbers on either side."""
    vocab, rows = 4001, 64
    h = handle(vocab)
    g = np.random.default_rng(11)
    tiny = np.array([0.0, -0.0, 1e-45, -1e-45, 3e-45, -3e-45, 1e-38, -1e-38, 2e-3, -2e-3, 5e-39], np.float32)
    x = tiny[g.integers(0, len(tiny), (rows, vocab))]
    x[::2, :40] = g.standard_normal((rows // 2, 40))
    T = np.exp(g.uniform(np.log(1e-3), 0, rows)).astype(np.float32)
    for filters in ("k", "p", "kpq"):
        k = g.integers(1, vocab, rows).astype(np.int32) if "k" in filters else None
        p = g.uniform(0, 1, rows).astype(np.float32) if "p" in filters else None
        q = np.exp(g.uniform(-5, 0, rows)).astype(np.float32) if "q" in filters else None
        u = g.uniform(0, 1, rows).astype(np.float32) * np.float32(1 - 2 ** -24)
        logits = torch.from_numpy(x).cuda()
        token, prob, status = sample(h, logits, u, T, k, p, q)
        assert status == 0
        verify(logits, T, k, p, q, u, token, prob)
    h.close()


def test_extreme_values():
    """Masks of the type's lowest value, logits of any size, temperatures from nothing
    to infinite, one logit left, u at both ends."""
    vocab = 3001
    h = handle(vocab)
    g = np.random.default_rng(5)
    low = np.finfo(np.float32).min
    base = g.standard_normal(vocab).astype(np.float32)
    rows, T = [], []
    for scale, t in ((1, 1), (1e30, 1e30), (1e30, 1e29), (1e-30, 1e-30), (1e-38, 1e-30), (1, 1e-30), (1, 1e30), (3e4, 1e4),
                     (1, 1e-38), (1e6, 0.01), (1, 3e38)):
        rows.append(base * np.float32(scale))
        T.append(t)
    masked = base.copy()
    masked[g.uniform(size=vocab) < 0.9] = low
    rows += [masked, np.full(vocab, low, np.float32), np.full(vocab, -np.inf, np.float32), base + np.float32(1e5)]
    rows[-2][1234] = -7.0
    one = np.full(vocab, low, np.float32)
    one[vocab - 1] = 3e38
    rows.append(one)
    T += [0.5, 0.5, 0.5, 0.5, 0.5]
    x, T = np.stack(rows), np.array(T, np.float32)
    n = len(T)
    logits = torch.from_numpy(x).cuda()
    for u in (0.0, 0.37, 1 - 2.0 ** -24):
        for k, p, q in ((None, None, None), (np.full(n, 17), np.full(n, 0.8), np.full(n, 0.01)),
                        (None, np.full(n, 0.0), None), (np.full(n, 1), None, None), (None, None, np.full(n, 2.0))):
            us = np.full(n, u, np.float32)
            token, prob, status = sample(h, logits, us, T, k, p, q)
            assert status == 0
            verify(logits, T, k, p, q, us, token, prob)
    h.close()


@pytest.mark.parametrize("vocab", [100, 50000])
def test_rows_that_are_refused(vocab):
    """Their token is -1 and their probability NaN; the others are as ever."""
    E, _ = _lib()
    h = handle(vocab)
    logits, g = make(12, vocab, seed=9, banned=0)
    T, _, p, q, u = params(g, 12, vocab, "pq")
    T, p, q = T.copy(), p.copy(), q.copy()
    for kind in range(9):
        x, t, pp, qq, uu = logits.clone(), T.copy(), p.copy(), q.copy(), u.copy()
        want = E.EBD_ERR_INVALID_ARG if kind > 3 else E.EBD_ERR_NONFINITE
        if kind == 0:
            x[4, vocab - 1] = float("nan")
        elif kind == 1:
            x[4, 0] = -float("nan")
        elif kind == 2:
            x[4, vocab // 2] = float("inf")
        elif kind == 3:
            x[4] = -float("inf")
        elif kind == 4:
            t[4] = -1
        elif kind == 5:
            t[4] = np.inf
        elif kind == 6:
            uu[4] = 1.0
        elif kind == 7:
            pp[4] = np.nan
        else:
            qq[4] = np.nan
        token, prob, status = sample(h, x, uu, t, None, pp, qq)
        assert status == want and token[4] == -1 and np.isnan(prob[4])
        ok = np.arange(12) != 4
        verify(x[torch.from_numpy(ok).cuda()], t[ok], None, pp[ok], qq[ok], uu[ok], token[ok], prob[ok])
        assert h.sync_status() == 0
    h.close()


@pytest.mark.parametrize("vocab,rows", [(700, 3), (40000, 3), (152064, 30), (152064, 90)])
def test_settings_at_their_ends(vocab, rows):
    """Equal logits under top-k of few, u = -0, filters that are infinite, -0 or of one
    token: each row its own."""
    h = handle(vocab)
    g = np.random.default_rng(8)
    x = np.zeros((rows, vocab), np.float32)
    x[1::3] = np.round(g.standard_normal((len(x[1::3]), vocab)) * 2) / 2
    x[2::3, :5] = 1.0
    T = np.full(rows, 0.9, np.float32)
    inf = np.inf
    k = g.choice([1, 2, 7, 300, 0, -5, 2 ** 31 - 1], rows).astype(np.int32)
    p = g.choice([-inf, -0.0, 0.3, 1.0, inf], rows).astype(np.float32)
    q = g.choice([-inf, -0.0, 0.5, 1.0, inf], rows).astype(np.float32)
    u = g.choice([-0.0, 0.25, 1 - 2.0 ** -24], rows).astype(np.float32)
    logits = torch.from_numpy(x).cuda()
    token, prob, status = sample(h, logits, u, T, k, p, q)
    assert status == 0
    verify(logits, T, np.maximum(k, 0), np.maximum(p, 0), np.maximum(q, 0), np.abs(u), token, prob)
    h.close()


@pytest.mark.parametrize("rows", [9, 200])
def test_top_p_where_bins_mislead(rows):
    """Logits at the near ends of their bins of (m - l) / T above a border and at the far
    ends below, and the other way round: weights taken as in the middle of their bins put
    the border half a bin's width of weights off, in another bin."""
    vocab = 152064
    h = handle(vocab)
    width = 40 / 2040  # of a bin, in powers of two, where masked logits are everywhere
    g = np.random.default_rng(12)
    x = np.full((rows, vocab), -np.inf, np.float32)
    p = np.empty(rows, np.float32)
    for r in range(rows):
        near = 0.45 if r % 2 else -0.45
        bins = np.repeat(np.arange(10, 50), 1900)
        y = (bins + np.where(bins < 30, near, -near)) * width
        l = np.concatenate([[0.0], -y * np.log(2)]).astype(np.float32)
        at = g.permutation(vocab)[: len(l)]
        x[r, at] = l
        w = np.exp(l.astype(np.float64))
        border = w[: 1 + 20 * 1900].sum() / w.sum()  # between the two kinds
        p[r] = border + (r // 2 % 5 - 2) * 1.2e-3
    u = g.uniform(0, 1, rows).astype(np.float32) * np.float32(1 - 2 ** -24)
    u[::3] = np.float32(1 - 2.0 ** -24)
    logits = torch.from_numpy(x).cuda()
    token, prob, status = sample(h, logits, u, None, None, p, None)
    assert status == 0
    verify(logits, None, None, p, None, u, token, prob)
    h.close()


def test_calls_on_streams_of_their_own():
    """Calls of several handles at once."""
    E, rt = _lib()
    vocab, rows = 60000, 40
    hs = [handle(vocab) for _ in range(4)]
    sets = []
    for i in range(4):
        logits, g = make(rows, vocab, seed=20 + i)
        T, k, p, q, u = params(g, rows, vocab, "kpq")
        dev = [_dev(u, torch.float32), _dev(T, torch.float32), _dev(k, torch.int32), _dev(p, torch.float32), _dev(q, torch.float32)]
        token, prob = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, **F32)
        a = E.ebd_sample_args()
        a.rows, a.logits, a.token, a.prob = rows, logits.data_ptr(), token.data_ptr(), prob.data_ptr()
        a.u, a.temperature, a.top_k, a.top_p, a.min_p = (t.data_ptr() for t in dev)
        sets.append((logits, T, k, p, q, u, token, prob, a, dev))
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(sets):
            E.check(E.ebd_sample(hs[i].h, s[8], rt.stream_handle(streams[i])), hs[i].h)
    torch.cuda.synchronize()
    for logits, T, k, p, q, u, token, prob, _, _ in sets:
        verify(logits, T, k, p, q, u, token.cpu().numpy(), prob.cpu().numpy())
    for h in hs:
        assert h.sync_status() == 0
        h.close()


def test_every_token_of_a_small_row():
    """u over a fine grid: every token comes up as often as its probability says."""
    vocab, n = 9, 512
    h = handle(vocab)
    l = torch.tensor([0.3, -1.0, 2.0, 2.0, -np.inf, 0.3, 1.1, -4.0, 0.0], device="cuda").repeat(n, 1)
    u = (np.arange(n) / n).astype(np.float32)
    token, prob, status = sample(h, l, u, np.full(n, 0.8))
    assert status == 0 and (np.diff(token) >= 0).all()
    verify(l, np.full(n, 0.8, np.float32), None, None, None, u, token, prob)
    want = torch.softmax(l[0].double() / float(np.float32(0.8)), 0).cpu().numpy()
    np.testing.assert_allclose(np.bincount(token, minlength=vocab) / n, want, atol=1.0 / n)
    h.close()


def test_refused_arguments():
    E, rt = _lib()
    h = handle(100, 8)
    t = torch.zeros((8, 100), **F32)
    v = torch.zeros((8,), **F32)

    def call(**over):
        a = E.ebd_sample_args()
        a.rows, a.logits, a.u, a.token, a.prob = 8, t.data_ptr(), v.data_ptr(), v.data_ptr(), v.data_ptr()
        for name, x in over.items():
            setattr(a, name, x)
        return E.ebd_sample(h.h, a, rt.stream_handle(None))

    for over in (dict(rows=9), dict(rows=-1), dict(dtype=3), dict(stride=99), dict(stride=-100), dict(logits=0), dict(u=0),
                 dict(token=0), dict(prob=0), dict(logits=t.data_ptr() + 2)):
        assert call(**over) == E.EBD_ERR_INVALID_ARG, over
    assert call(rows=0, logits=0) == E.EBD_OK
    assert E.ebd_sample(None, E.ebd_sample_args(), 0) == E.EBD_ERR_INVALID_ARG
    torch.cuda.synchronize()
    h.close()


def test_in_a_graph_and_on_another_stream():
    """A captured call draws by what its buffers hold when it is replayed."""
    E, rt = _lib()
    vocab, rows = 30011, 6
    h = handle(vocab)
    buf = torch.zeros((rows, vocab), **F32)
    u, T = torch.zeros((rows,), **F32), torch.full((rows,), 0.9, **F32)
    p = torch.full((rows,), 0.9, **F32)
    token, prob = torch.zeros((rows,), dtype=torch.int32, device="cuda"), torch.zeros((rows,), **F32)
    a = E.ebd_sample_args()
    a.rows, a.logits, a.u, a.temperature, a.top_p = rows, buf.data_ptr(), u.data_ptr(), T.data_ptr(), p.data_ptr()
    a.token, a.prob = token.data_ptr(), prob.data_ptr()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        E.check(E.ebd_sample(h.h, a, rt.stream_handle(None)), h.h)
    for seed in range(3):
        logits, g = make(rows, vocab, seed=seed)
        buf.copy_(logits)
        uu = g.uniform(0, 1, rows).astype(np.float32) * np.float32(1 - 2 ** -24)
        u.copy_(torch.from_numpy(uu))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        assert h.sync_status(s) == 0
        verify(buf, np.full(rows, 0.9, np.float32), None, np.full(rows, 0.9, np.float32), None, uu, token.cpu().numpy(),
               prob.cpu().numpy())
    h.close()
