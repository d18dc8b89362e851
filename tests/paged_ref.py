"""The paged K/V cache in 64 bits, and a cache with its calls on the GPU
(tests): e4m3 rows by their definition, attention row by row."""
from __future__ import annotations

import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if (e, m) == (15, 7) else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        out[c] = -x if c & 128 else x
    return out


def quantise(x: np.ndarray):
    """Codes and exponent bytes of rows x [..., D] (float64 of bf16 values)."""
    x = np.asarray(x, np.float64)
    fin = np.isfinite(x)
    amax = np.abs(np.where(fin, x, 0)).max(-1)
    # the least k >= -127 with amax <= 448 * 2^k: frexp gives amax = f * 2^e, f in [0.5, 1)
    f, e = np.frexp(amax)
    k = np.where(amax == 0, -127, np.maximum(e - 9 + (f > 0.875), -127))
    y = np.ldexp(np.where(fin, x, 0), -k[..., None])
    y = np.where(k[..., None] == 120, np.clip(y, -240, 240), y)  # 256 * 2^120 is no bf16 value
    a = np.abs(y)
    q = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))     # binade; below 2^-6 the grid is 2^-9
    n = np.rint(np.ldexp(a, (3 - q).astype(int)))       # half to even, 8..16 (0..8 below)
    up = n == 16
    q, n = q + up, np.where(up, 8, n)
    code = np.where(n < 8, n, (q + 7) * 8 + (n - 8)).astype(np.int64)
    code = np.where(np.signbit(x), code | 128, code)
    row = fin.all(-1)
    return (np.where(row[..., None], code, 0x7F).astype(np.uint8),
            np.where(row, k + 127, 255).astype(np.uint8))


def dequantise(code, e):
    x = np.ldexp(e4m3_values()[code], np.minimum(e.astype(np.int64), 247)[..., None] - 127)
    return np.where(e[..., None] == 255, np.nan, x)


def attend(q, k, v, lens, kv_lens, group, causal, scale):
    """q [R][Hq][D]; k, v: per sequence [len][Hkv][D]; float64 tensors.
    Returns the output and how far a bf16 result may be from it.  Rounding to
    bf16 (8 significant bits: half a step is 2^-8 of the value at most) moves a
    probability by 2^-8 of itself, so an element by 2^-8 sum p|v| / sum p, and
    the output by 2^-8 of itself.  A score is a sum of D products in
    32 bits, of up to 16 roundings, and q in two 4-bit terms loses less than
    2^-18 of its largest element: together below 2^-17 of S = scale sum |q||k|,
    by which a probability is then off.  The exponential and the sums over keys
    stay below 2^-12 of sum p|v| / sum p."""
    import torch
    out, tol = torch.zeros_like(q), torch.full_like(q, 1e-30)
    r = 0
    for n, m, kk, vv in zip(lens, kv_lens, k, v):
        for i in range(n):
            see = max(0, min(m, m - n + i + 1)) if causal else m
            if see == 0:
                continue
            qi = q[r + i].view(-1, group, q.shape[-1])                       # [Hkv][G][D]
            s = torch.einsum("hgd,khd->hgk", qi, kk[:see]) * scale
            top = abs(scale) * torch.einsum("hgd,khd->hgk", qi.abs(), kk[:see].abs()).amax(-1, keepdim=True)
            p = torch.softmax(s, -1)
            o = torch.einsum("hgk,khd->hgd", p, vv[:see])
            mag = torch.einsum("hgk,khd->hgd", p, vv[:see].abs())
            out[r + i] = o.reshape(q.shape[1:])
            tol[r + i] = (2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -17 * top) * mag).reshape(q.shape[1:]) + 1e-30
        r += n
    return out, tol


class Cache:
    """Pools, a page table with pages in random order, and the calls."""

    def __init__(self, heads, dtype, page, lens, *, seed=0, spare=2, interleaved=False, cover=None):
        import torch
        self.torch = torch
        self.hq, self.hkv, self.D = heads
        self.dtype, self.page, self.B = dtype, page, len(lens)
        rng = np.random.default_rng(seed)
        need = [(n + page - 1) // page for n in (cover or lens)]
        self.n_pages = sum(need) + spare
        self.max_pages = max(need + [1])
        perm = rng.permutation(self.n_pages)
        table = np.full((max(self.B, 1), self.max_pages), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = perm[at: at + n]
            at += n
        self.table_h = table
        self.table = torch.from_numpy(table).cuda()
        el = torch.uint8 if dtype == "e4m3" else torch.bfloat16
        per = self.hkv * page * self.D
        if interleaved:  # K and V of a page side by side in one buffer
            buf = torch.zeros((self.n_pages, 2, self.hkv, page, self.D), dtype=el, device="cuda")
            self.k, self.v, self.stride = buf[:, 0], buf[:, 1], 2 * per
        else:
            self.k = torch.zeros((self.n_pages, self.hkv, page, self.D), dtype=el, device="cuda")
            self.v = torch.zeros_like(self.k)
            self.stride = 0
        self.ks = self.vs = None
        if dtype == "e4m3":
            self.ks = torch.zeros((self.n_pages, self.hkv, page), dtype=torch.uint8, device="cuda")
            self.vs = torch.zeros_like(self.ks)

    def pages(self, E):
        c = E.ebd_kv_pages()
        c.k, c.v, c.page_table = self.k.data_ptr(), self.v.data_ptr(), self.table.data_ptr()
        if self.dtype == "e4m3":
            c.k_scale, c.v_scale, c.dtype = self.ks.data_ptr(), self.vs.data_ptr(), E.EBD_KV_E4M3
        c.page_stride, c.page_size = self.stride, self.page
        c.n_pages, c.max_pages = self.n_pages, self.max_pages
        return c

    def fill(self, k, v):
        """Every place of every page from bf16 tensors [n_pages][Hkv][page][D]."""
        torch = self.torch
        for pool, sc, x in ((self.k, self.ks, k), (self.v, self.vs, v)):
            if self.dtype == "bf16":
                pool.copy_(x)
            else:
                code, e = quantise(x.double().cpu().numpy())
                pool.copy_(torch.from_numpy(code))
                sc.copy_(torch.from_numpy(e))

    def value(self, which):
        """The pool in 64 bits, on the GPU."""
        torch = self.torch
        x = (self.k, self.v)[which]
        if self.dtype == "bf16":
            return x.double()
        tab = torch.from_numpy(e4m3_values()).cuda()
        e = (self.ks, self.vs)[which].double() - 127
        x = tab[x.long()] * torch.ldexp(torch.ones_like(e), e)[..., None]
        return torch.where(e[..., None] == 128, torch.full_like(x, math.nan), x)

    def rows_of(self, which, b, n):
        """Positions [0, n) of sequence b: [n][Hkv][D], 64 bits."""
        idx = self.torch.from_numpy(self.table_h[b, : (n + self.page - 1) // self.page].astype(np.int64)).cuda()
        if which not in self.__dict__.setdefault("_value", {}):
            self._value[which] = self.value(which)
        x = self._value[which][idx]                                          # [P][Hkv][page][D]
        return x.transpose(1, 2).reshape(-1, self.hkv, self.D)[:n]


def handle(E, rt, heads, batch, rows, paged=1):
    hq, hkv, D = heads
    return rt.Handle(E.ebd_config(
        d_model=64, vocab=64, n_heads_q=hq, n_heads_kv=hkv, head_dim=D, d_base=64,
        max_batch=max(batch, 1), max_window=1, max_rows=max(rows, 1), max_prefix=0, gen_len=1,
        g_max=5, l_min=8, l_b=32, eos_id=63, lps_enabled=1, tau=0.9, tau_psi=0.89, paged=paged))


def cu_rows(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
