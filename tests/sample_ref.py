"""Sampling in 64 bits, and what a drawn token may differ by.

A kernel's weights are off by 2^-30 of themselves and 2^-43 of the largest; sums of
them are exact, and so are the parts of them that a share or a random number takes, but
for a unit of 2^-43.  So a border lies within slack() of all that is kept from where it
is here: twice 2^-30, for what lies below it and for the whole, and twice 2^-43 for
every logit.  numpy's own are off by 2^-50 at
most at these sizes.
"""
import math

import numpy as np


def slack(w):
    """Of the sum of weights w (the largest of them 1)."""
    return 2.0 ** -29 + 2.0 ** -42 * (1 + np.count_nonzero(w)) / w.sum()


def order(l):
    """Indices by descending logit, the lower index first."""
    return np.argsort(-l, kind="stable")


def kept(l, T, k=0, p=1.0, q=0.0, shift=0.0):
    """Indices that are kept, in the order; the share p moved by `shift`."""
    m = l.max()
    x = (l - m) / T
    w = np.where(x < -40 * math.log(2.0), 0.0, np.exp(np.maximum(x, -1e4)))
    idx = order(l)
    if k > 0:
        idx = idx[:k]
    if p < 1:
        c = np.cumsum(w[idx])
        idx = idx[: int((c < (p + shift) * c[-1]).sum()) + 1]
    if q > 0:
        idx = idx[x[idx] >= math.log(min(q, 1.0))]
    return idx, w


def check(l, T, u, token, prob, k=0, p=1.0, q=0.0):
    """Whether `token` and `prob` are right for logits l (any float array)."""
    l = np.asarray(l, np.float64)
    T, u, p, q = (float(np.float32(v)) for v in (T, u, p, q))
    if T == 0:
        assert token == int(np.argmax(l)) and prob == 1.0
        return
    T = min(max(T, float(np.float32(1e-30))), float(np.float32(1e30)))
    why = None
    eps = slack(kept(l, T, k)[1])  # of the row's sum, which p's share is taken of
    for shift in (0.0, -eps, eps):
        idx, w = kept(l, T, k, p, q, shift)
        idx = np.sort(idx)
        c = np.cumsum(w[idx])
        total = c[-1]
        eps = max(eps, slack(w[idx]))
        at = np.searchsorted(idx, token)
        if at >= len(idx) or idx[at] != token:
            why = f"token {token} is not kept"
            continue
        lo = c[at - 1] if at else 0.0
        if not lo - eps * total <= u * total <= c[at] + eps * total:
            why = f"u points at {idx[np.searchsorted(c, u * total, side='right')]}, not at {token}"
            continue
        want = w[token] / total
        # rounded to 32 bits, and the sum off by eps; w itself is computed in 64 bits
        assert abs(prob - want) <= want * (2.0 ** -24 + 2 * eps), (prob, want)
        return
    raise AssertionError(why)
