"""The work that programs have the paged K/V cache do, as measured cases.

A server that keeps the K/V of many sequences of unequal length holds them in
pages of a few positions, in bf16 or in 8 bits (e4m3 with one power-of-two
scale per position and head).  It calls three operators: `ebd_paged_write`
quantises rows of new tokens into the pages, `ebd_paged_attention` lets the
rows of a chunk of new tokens, or single tokens, attend to everything that a
sequence has in its pages, and `ebd_paged_read` reads rows back as bf16 (a
cache that is swapped out, or handed to the dense-cache step).

The sizes are this repository's own (the tiny, LLaDA-8B and Dream-7B heads of
`synth/configs.py`, windows of 1 to 64 rows, up to 64 sequences, prefixes up to
4096) and, beyond its dense cache, generic: prompts taken in chunks and long
contexts.  `draw` spreads over the same ranges.

Values: K channels of unequal size and V heads of unequal size (what a scale
per position and head is there for), query heads of unequal sharpness, so that
some rows attend to a few keys and some to all.  Pages are handed out in random
order; what a page holds past its sequence's end is another sequence's.
"""
from __future__ import annotations

import math

import torch

own = False

# query heads, K/V heads, head width
TINY = (4, 4, 64)
LLADA_8B = (32, 32, 128)
DREAM_7B = (28, 4, 128)


def _case(entry, heads, dtype, page, batch, new, ctx, *, ragged=False, causal=False, fused=False,
          skip=False, name=None):
    c = dict(entry=entry, heads_q=heads[0], heads_kv=heads[1], head_dim=heads[2], dtype=dtype,
             page=page, batch=batch, new=new, ctx=ctx, ragged=ragged, causal=causal, fused=fused,
             skip=skip)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's step: the committed rows of a window go into the cache
        _case("write", LLADA_8B, "e4m3", 64, 1, 32, 512, skip=True, name="write_window"),
        # a batch's windows, ragged, out of the fused projection's rows, into small pages
        _case("write", DREAM_7B, "bf16", 16, 64, 48, 1024, ragged=True, fused=True,
              name="write_batch"),
        # prompts enter the cache
        _case("write", LLADA_8B, "e4m3", 64, 8, 512, 0, name="write_prompt"),
        # one window read back
        _case("read", TINY, "bf16", 16, 1, 64, 100, name="read_window"),
        # four sequences swapped out
        _case("read", LLADA_8B, "e4m3", 64, 4, 1024, 0, name="read_swap"),
        # the smallest attention: latency
        _case("attend", TINY, "bf16", 16, 1, 32, 128, name="attend_tiny"),
        # one user's window over its prefix
        _case("attend", LLADA_8B, "e4m3", 64, 1, 32, 512, name="attend_window"),
        # single tokens of many users, grouped heads, 8-bit cache
        _case("attend", DREAM_7B, "e4m3", 64, 64, 1, 4096, ragged=True, causal=True, fused=True,
              name="attend_tokens"),
        # single tokens of some users, a K/V head per query head, bf16, small pages
        _case("attend", LLADA_8B, "bf16", 16, 16, 1, 2011, ragged=True, causal=True,
              name="attend_tokens_mha"),
        # batched serving: windows of many sequences
        _case("attend", LLADA_8B, "e4m3", 32, 64, 32, 1024, ragged=True, name="attend_windows"),
        # two prompts' next chunks, causal
        _case("attend", DREAM_7B, "bf16", 64, 2, 1000, 7000, causal=True, fused=True,
              name="attend_chunk"),
        # a window over one long document
        _case("attend", DREAM_7B, "e4m3", 128, 1, 61, 60000, name="attend_long"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


MAX_ROWS = 4096        # rows of a call
MAX_BYTES = 5.7e8      # cache that an attention reads, at most (attend_windows)
MAX_FLOPS = 2.1e11     # and what it computes, at most (attend_chunk)


def draw(rng):
    if rng.random() < 0.6:
        heads = rng.choice((TINY, LLADA_8B, LLADA_8B, DREAM_7B, DREAM_7B))
    else:
        hkv = rng.choice((1, 2, 4, 8))
        heads = (hkv * rng.choice((1, 2, 4, 7, 8)), hkv, rng.choice((64, 128)))
    dtype = rng.choice(("bf16", "e4m3"))
    page = rng.choice((16, 32, 64, 128))
    flags = dict(ragged=rng.random() < 0.6, fused=rng.random() < 0.4)
    entry = rng.choice(("attend", "attend", "attend", "write", "read"))
    if entry != "attend":
        batch = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, min(1024, MAX_ROWS // batch))
        return _case(entry, heads, dtype, page, batch, new, _log_int(rng, 1, 1024),
                     skip=entry == "write" and rng.random() < 0.5, **flags)
    batch = _log_int(rng, 1, 64)
    kind = rng.choice(("token", "window", "window", "chunk"))
    new = {"token": 1, "window": rng.randint(2, 64), "chunk": rng.randint(65, 1024)}[kind]
    new = min(new, MAX_ROWS // batch)
    per_key = batch * heads[1] * heads[2] * 2 * (1 if dtype == "e4m3" else 2)
    per_pair = 4 * batch * new * heads[0] * heads[2]
    top = int(min(65536, MAX_BYTES / per_key - new, MAX_FLOPS / per_pair - new))
    ctx = _log_int(rng, 16, max(16, top))
    return _case(entry, heads, dtype, page, batch, new, ctx,
                 causal=kind != "window" or rng.random() < 0.2, **flags)


# ------------------------------------------------------------------ inputs
def _lens(case):
    """New rows and cached positions before them, of every sequence (host
    lists); a ragged case's are part of the case, so that its outputs keep
    their shapes."""
    b, n, p = case["batch"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [n] * b, [p] * b
    g = torch.Generator().manual_seed(b * 8191 + n * 131 + p)
    ns = torch.randint(max(1, n // 4), n + 1, (b,), generator=g).tolist()
    ps = torch.randint(p // 2, p + 1, (b,), generator=g).tolist()
    return ns, ps


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + what * 7919 + 17) % (1 << 62))


def _normal(seed, what, shape):
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    return x.normal_(0.0, 1.0, generator=_gen(seed, what))


def _uniform(seed, what, shape, lo, hi):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(lo, hi, generator=_gen(seed, what))


def _quantise(x):
    """e4m3 codes of rows x [..., D] and the exponent byte e of their scale
    2^(e-127): the least power of two with amax <= 448 * scale (at the largest,
    codes stop at 240: 256 * 2^120 is past bf16's range).  A row with a value
    that is not finite is NaN as a whole: e = 255, codes 0x7F."""
    x = x.float()
    finite = torch.isfinite(x).all(-1)
    bits = x.abs().amax(-1).view(torch.int32)
    e = (bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()
    e = torch.where(finite, e.clamp(min=0), torch.full_like(e, 255))
    inv = ((254 - e.clamp(max=247)) << 23).view(torch.float32)
    top = torch.where(e == 247, torch.full_like(inv, 240.0), torch.full_like(inv, 448.0))[..., None]
    code = torch.minimum(torch.maximum(x * inv[..., None], -top), top).to(torch.float8_e4m3fn).view(torch.uint8)
    return torch.where(finite[..., None], code, torch.full_like(code, 0x7F)), e.to(torch.uint8)


def _scale_of(e):
    """2^(e-127) of exponent bytes."""
    e = e.to(torch.int32)
    return torch.where(e > 0, e << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


class _State:
    """What a program holds: the cache, its page table, the call's rows."""


def prepare(case, seed):
    hq, hkv, hd, page = (case[k] for k in ("heads_q", "heads_kv", "head_dim", "page"))
    ns, ps = _lens(case)
    b, n = case["batch"], sum(ns)
    s = _State()
    s.case, s.longest = case, max(ns)
    dev = dict(device="cuda")
    i32 = dict(dtype=torch.int32, **dev)
    # pages in random order, some to spare; a sequence's entries past its own pages are -1
    need = [(p + w + page - 1) // page for w, p in zip(ns, ps)]
    s.n_pages = sum(need) + 2
    order = torch.randperm(s.n_pages, generator=torch.Generator().manual_seed(seed % (1 << 62))).tolist()
    s.table = torch.full((b, max(need)), -1, dtype=torch.int32)
    for i, k in enumerate(need):
        s.table[i, :k] = torch.tensor(order[:k], dtype=torch.int32)
        order = order[k:]
    s.table = s.table.cuda()
    cu = [0]
    for w in ns:
        cu.append(cu[-1] + w)
    s.cu_rows = torch.tensor(cu, **i32)
    s.kv_len = torch.tensor([w + p for w, p in zip(ns, ps)], **i32)
    first = ps if case["entry"] != "read" else [0] * b
    s.row_pos = torch.cat([torch.arange(f, f + w, dtype=torch.int32) for w, f in zip(ns, first)]).cuda()
    s.skip = None
    if case["skip"]:
        s.skip = (_uniform(seed, 1, (n,), 0, 1) < 0.6).to(torch.uint8)
    # the cache
    k_gain = torch.exp(_uniform(seed, 2, (hkv, 1, hd), -1.2, 0.8))
    v_gain = torch.exp(_uniform(seed, 3, (hkv, 1, 1), -2.0, 2.0))
    s.pools, s.scales = [], []
    for what, gain in ((4, k_gain), (5, v_gain)):
        x = _normal(seed, what, (s.n_pages, hkv, page, hd))
        x.mul_(gain.bfloat16())
        e = None
        if case["dtype"] == "e4m3":
            code = torch.empty(x.shape, dtype=torch.uint8, **dev)
            e = torch.empty(x.shape[:-1], dtype=torch.uint8, **dev)
            step = max(1, (1 << 27) // (hkv * page * hd))
            for i in range(0, s.n_pages, step):
                code[i: i + step], e[i: i + step] = _quantise(x[i: i + step])
            x = code
        s.pools.append(x)
        s.scales.append(e)
    # the rows of the call: slices of one buffer where the projection is fused
    q_gain = torch.exp(_uniform(seed, 6, (hq, 1), -0.7, 1.2)).bfloat16()
    qkv = _normal(seed, 7, (n, hq + 2 * hkv, hd))
    qkv[:, :hq].mul_(q_gain)
    qkv[:, hq: hq + hkv].mul_(k_gain.bfloat16().view(1, hkv, hd))
    qkv[:, hq + hkv:].mul_(v_gain.bfloat16().view(1, hkv, 1))
    q, k, v = qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
    if not case["fused"]:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    s.q, s.k, s.v = q, k, v
    if case["entry"] == "read":
        s.k, s.v = torch.zeros_like(k), torch.zeros_like(v)
    s.out = torch.zeros((n, hq, hd), dtype=torch.bfloat16, **dev)
    if own:
        _prepare_own(s, case, n)
    torch.cuda.synchronize()
    return s


def _prepare_own(s, case, n):
    """The handle and the argument structures that a program keeps."""
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    hq, hkv, hd = (case[k] for k in ("heads_q", "heads_kv", "head_dim"))
    s.E, s.rt = E, rt
    s.handle = rt.Handle(E.ebd_config(
        d_model=hq * hd, vocab=4096, n_heads_q=hq, n_heads_kv=hkv, head_dim=hd, d_base=hq * hd,
        max_batch=case["batch"], max_window=64, max_rows=n, max_prefix=0, gen_len=64, g_max=5,
        l_min=8, l_b=32, eos_id=4095, lps_enabled=1, tau=0.9, tau_psi=0.89, paged=1))
    c = s.cache = E.ebd_kv_pages()
    c.k, c.v = (t.data_ptr() for t in s.pools)
    if case["dtype"] == "e4m3":
        c.dtype = E.EBD_KV_E4M3
        c.k_scale, c.v_scale = (t.data_ptr() for t in s.scales)
    c.page_table, c.max_pages = s.table.data_ptr(), s.table.shape[1]
    c.page_size, c.n_pages = case["page"], s.n_pages
    a = s.args = E.ebd_paged_args()
    a.batch, a.rows, a.max_new = case["batch"], n, s.longest
    a.cu_rows, a.row_pos, a.kv_len = s.cu_rows.data_ptr(), s.row_pos.data_ptr(), s.kv_len.data_ptr()
    a.q, a.k, a.v, a.out = s.q.data_ptr(), s.k.data_ptr(), s.v.data_ptr(), s.out.data_ptr()
    a.q_stride, a.kv_stride = s.q.stride(0), s.k.stride(0)
    a.skip = s.skip.data_ptr() if s.skip is not None else None
    a.causal = int(case["causal"])
    s.call = {"write": E.ebd_paged_write, "read": E.ebd_paged_read,
              "attend": E.ebd_paged_attention}[case["entry"]]


# ------------------------------------------------------------------ one pass
def run(s):
    if own:
        h = s.handle.h
        s.E.check(s.call(h, s.cache, s.args, s.rt.stream_handle(None)), h)
    elif s.case["entry"] == "write":
        _plain_write(s)
    elif s.case["entry"] == "read":
        s.k, s.v = _plain_read(s)
    else:
        s.out = _plain_attend(s)
    if s.case["entry"] == "attend":
        return s.out
    if s.case["entry"] == "read":
        return {"k": s.k, "v": s.v}
    if s.case["dtype"] == "bf16":
        return {"k": s.pools[0], "v": s.pools[1]}
    # 8-bit values, and their scales' exponents as whole numbers
    return {"k": s.pools[0].view(torch.float8_e4m3fn), "v": s.pools[1].view(torch.float8_e4m3fn),
            "k_scale": s.scales[0], "v_scale": s.scales[1]}


def _row_slots(s):
    """Sequence, page and place in the page of every row of the call."""
    rows = torch.arange(s.row_pos.numel(), device="cuda")
    seq = torch.searchsorted(s.cu_rows[1:].long(), rows, right=True)
    pos = s.row_pos.long()
    page = s.case["page"]
    return rows, seq, s.table[seq, pos // page].long(), pos % page


def _plain_write(s):
    _, _, pg, off = _row_slots(s)
    keep = torch.ones(pg.shape, dtype=torch.bool, device="cuda") if s.skip is None else s.skip == 0

    def put(pool, new):
        wide = keep.view((-1,) + (1,) * (new.dim() - 1))
        pool[pg, :, off] = torch.where(wide, new, pool[pg, :, off])

    if s.case["dtype"] == "bf16":
        put(s.pools[0], s.k), put(s.pools[1], s.v)
        return
    (kc, ke), (vc, ve) = _quantise(s.k), _quantise(s.v)
    put(s.pools[0], kc), put(s.pools[1], vc)
    put(s.scales[0], ke), put(s.scales[1], ve)


def _values(s, which, at):
    """Cache entries at an index, in 32 bits."""
    x = s.pools[which][at]
    if s.case["dtype"] == "bf16":
        return x.float()
    return x.view(torch.float8_e4m3fn).float() * _scale_of(s.scales[which][at])[..., None]


def _plain_read(s):
    _, _, pg, off = _row_slots(s)
    at = (pg, slice(None), off)
    return _values(s, 0, at).bfloat16(), _values(s, 1, at).bfloat16()


def _plain_attend(s):
    c = s.case
    hq, hkv, hd, b, n = c["heads_q"], c["heads_kv"], c["head_dim"], c["batch"], s.longest
    g = hq // hkv
    pages = s.table.clamp(min=0).long()
    keys = pages.shape[1] * c["page"]
    k, v = (_values(s, i, pages).permute(0, 2, 1, 3, 4).reshape(b, hkv, keys, hd) for i in (0, 1))
    cu, t = s.cu_rows.long(), torch.arange(n, device="cuda")
    new = cu[1:] - cu[:-1]
    at = (cu[:-1, None] + t).clamp(max=s.q.shape[0] - 1)
    q = s.q[at].float().view(b, n, hkv, g, hd).permute(0, 2, 3, 1, 4).reshape(b, hkv, g * n, hd)
    # row i of a sequence of m new rows sees its keys before kv_len, or, where
    # causal, before kv_len - m + i + 1
    last = s.kv_len.long()[:, None].expand(b, n)
    if c["causal"]:
        last = last - new[:, None] + t + 1
    hidden = torch.arange(keys, device="cuda") >= last[..., None]
    p = ((q @ k.transpose(2, 3)) * (1.0 / math.sqrt(hd))).view(b, hkv, g, n, keys)
    p.masked_fill_(hidden[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    p.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    z = p.sum(-1, keepdim=True)
    o = (p.view(b, hkv, g * n, keys) @ v).view(b, hkv, g, n, hd)
    o = torch.where(z > 0, o / z, torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(b, n, hq, hd)
    rows, seq, _, _ = _row_slots(s)
    return o[seq, rows - cu[seq]].bfloat16()


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    hq, hkv, hd = (case[k] for k in ("heads_q", "heads_kv", "head_dim"))
    ns, ps = _lens(case)
    n = sum(ns)
    # bytes of one position's K and V in the cache
    held = 2.0 * hkv * (hd + 1 if case["dtype"] == "e4m3" else 2 * hd)
    if case["entry"] != "attend":
        kept = 0.4 if case["skip"] else 1.0
        return {"bytes": n * (kept * (held + 4.0 * hkv * hd) + 8.0), "flops": 4.0 * n * hkv * hd}
    nbytes, flops = 4.0 * n * hq * hd, 0.0
    for w, p in zip(ns, ps):
        nbytes += (p + w) * held
        pairs = w * p + (w * (w + 1) / 2 if case["causal"] else w * w)
        flops += 4.0 * pairs * hq * hd
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------ the same in 64 bits
def _e4m3_table():
    """The value of each of the 256 codes."""
    out = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if e == 15 and m == 7 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out.append(-x if c & 128 else x)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _pow2(k):
    """2^k of whole k, exactly (pow is off by a last bit at some k)."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x):
    """Values of the codes (without the scale) that rows x become."""
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(amax / 448.0)).clamp(min=-127)
    k = torch.where(448.0 * _pow2(k - 1) >= amax, k - 1, k)
    k = torch.where(448.0 * _pow2(k) < amax, k + 1, k)
    y = x / _pow2(k)
    grid = _pow2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / grid) * grid


def _exact_pool(s, which, at):
    x = s.pools[which][at]
    if s.case["dtype"] == "bf16":
        return x.double()
    e = s.scales[which][at].double()
    return _e4m3_table()[x.long()] * _pow2(e - 127)[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    ns, ps = _lens(case)
    cu, pos, table = s.cu_rows.tolist(), s.row_pos.tolist(), s.table.tolist()
    page, hd, hkv = case["page"], case["head_dim"], case["heads_kv"]
    if case["entry"] in ("write", "read"):
        pg = torch.tensor([table[i][pos[r] // page] for i in range(case["batch"])
                           for r in range(cu[i], cu[i + 1])], device="cuda")
        off = torch.tensor([p % page for p in pos], device="cuda")
    if case["entry"] == "read":
        return {"k": _exact_pool(s, 0, (pg, slice(None), off)),
                "v": _exact_pool(s, 1, (pg, slice(None), off))}
    if case["entry"] == "write":
        kept = torch.arange(len(pos), device="cuda")
        if s.skip is not None:
            kept = kept[s.skip == 0]
        out = []
        for which, rows in ((0, s.k), (1, s.v)):
            x = s.pools[which]
            x = x.double() if case["dtype"] == "bf16" else _e4m3_table()[x.long()]
            new = rows.double() if case["dtype"] == "bf16" else _exact_codes(rows)
            x[pg[kept], :, off[kept]] = new[kept]
            out.append(x)
        return {"k": out[0], "v": out[1], "k_scale": None, "v_scale": None}
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    g = case["heads_q"] // hkv
    for i, (w, p) in enumerate(zip(ns, ps)):
        pages = s.table[i, : (w + p + page - 1) // page].long()
        k, v = (_exact_pool(s, j, pages).transpose(0, 1).reshape(hkv, -1, hd)[:, : w + p] for j in (0, 1))
        for h in range(case["heads_q"]):
            a = s.q[cu[i]: cu[i + 1], h].double() @ k[h // g].T / math.sqrt(hd)
            if case["causal"]:
                a += torch.full((w, w + p), -math.inf, dtype=torch.float64, device="cuda").triu(p + 1)
            out[cu[i]: cu[i + 1], h] = torch.softmax(a, -1) @ v[h // g]
    return out
