"""ebd_sample where its borders are hardest to find: shares close to 1, few tokens
allowed, the lowest logits, light tokens."""
import numpy as np
import pytest

from tests.test_gpu_sample import handle, make, sample, verify

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LAST = np.float32(1 - 2.0 ** -24)  # the last number below 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,rows", [(500, 24), (4096, 24), (4096, 200), (152064, 12), (152064, 90)])
def test_top_p_near_one(vocab, rows, dtype):
    """The share that is left out lies below all roundings of what bounds the sums by
    bins (10^-4): by itself, and of what top-k leaves."""
    h = handle(vocab)
    logits, g = make(rows, vocab, dtype, seed=vocab + rows)
    p = np.resize(np.array([0.9999, 0.99995, 0.99999, LAST], np.float32), rows)
    u = g.uniform(0, 1, rows).astype(np.float32) * LAST
    u[::3] = LAST
    T = np.exp(g.uniform(np.log(0.3), np.log(2), rows)).astype(np.float32)
    for k in (None, np.full(rows, vocab * 4 // 5, np.int32), np.full(rows, vocab // 40, np.int32)):
        for t in (None, T):
            token, prob, status = sample(h, logits, u, t, k, p)
            assert status == 0
            verify(logits, t, k, p, None, u, token, prob)
    h.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,rows", [(2000, 16), (4096, 200), (152064, 16), (152064, 90)])
def test_top_k_of_few_allowed(vocab, rows, dtype):
    """All but a few tokens banned, and fewer threads than k with one to show: what k asks
    for is then behind their largest, whether those are equal, nearly so, or one."""
    h = handle(vocab)
    allowed = [{8: 5.0, 10: 3.0}, {8: 5.0, 10: 3.0, vocab - 3: 5.0}, {9: 1.0, 11: 2.0, 1001: 2.0, 1003: -1.0, 1005: 2.0},
               {0: 2.0 ** -95, 2: 2.0 ** -96, 1000: 2.0 ** -95 + 2.0 ** -101}, {4: 0.0, 5: -1.0, 6: -2.0, 7: -0.5},
               {40: -3.0}, {vocab - 1: 1.0, vocab - 3: 0.5, vocab - 2: 0.0}, {i: float(i % 7) for i in range(0, 640, 2)}]
    x = np.full((rows, vocab), -np.inf, np.float32)
    T = np.ones(rows, np.float32)
    for r in range(rows):
        a = allowed[r % len(allowed)]
        x[r, list(a)] = list(a.values())
        if r % len(allowed) == 3:
            T[r] = 2.0 ** -96
    logits = torch.from_numpy(x).cuda().to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    g = np.random.default_rng(7)
    u = g.uniform(0, 1, rows).astype(np.float32) * LAST
    u[rows // 2:] = LAST
    for k in (2, 3, 10, 700):
        ks = np.full(rows, k, np.int32)
        for p in (None, g.uniform(0.3, 1, rows).astype(np.float32)):
            token, prob, status = sample(h, logits, u, T, ks, p)
            assert status == 0
            verify(logits, T, ks, p, None, u, token, prob)
    h.close()


@pytest.mark.parametrize("vocab", [8, 5000])
def test_min_p_below_the_lowest_logit(vocab):
    """Every logit is the type's lowest, and what min-p asks for lies below it: past
    float's range, where a share of equal logits is still kept by index."""
    h = handle(vocab)
    rows = 6
    logits = torch.full((rows, vocab), np.finfo(np.float32).min, device="cuda")
    T, q = np.full(rows, 1e30, np.float32), np.full(rows, 1e-7, np.float32)
    p = np.array([0.5, 0.25, 0.75, 0.5, 0.25, 0.75], np.float32)
    u = np.array([0, 0.5, LAST, LAST, 0.25, 0.5], np.float32)
    token, prob, status = sample(h, logits, u, T, None, p, q)
    assert status == 0
    verify(logits, T, None, p, q, u, token, prob)
    h.close()


@pytest.mark.parametrize("T", [1.0, 0.3, 1.7])
def test_weights_of_light_tokens(T):
    """The lighter of two tokens, from 2^-1 down to 2^-39 of the other: its probability is
    its weight, off by 2^-30 of itself, over a sum off by 2^-42 of the other's (twice a
    unit), rounded to 32 bits."""
    vocab, rows = 2, 500
    h = handle(vocab)
    g = np.random.default_rng(2)
    x = np.zeros((rows, vocab), np.float32)
    T = float(np.float32(T))
    x[:, 0] = -g.uniform(1, 39, rows) * np.log(2) * T
    for top in (0.0, 11.0, -3.7):
        l = (x + np.float32(top)).astype(np.float32)
        token, prob, status = sample(h, torch.from_numpy(l).cuda(), np.zeros(rows, np.float32), np.full(rows, T, np.float32))
        assert status == 0 and (token == 0).all()
        w = np.exp((l[:, 0].astype(np.float64) - l[:, 1]) / T)
        want = w / (1 + w)
        assert (np.abs(prob - want) <= want * (2.0 ** -24 + 2.0 ** -30 + 2.0 ** -42 + 2.0 ** -50)).all()
    h.close()
