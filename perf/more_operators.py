"""The work that a serving step does between its last hidden states and the
next step's cache, as measured cases.

`ebd_lm_logits` computes the logits of a step's rows, `ebd_sample` draws a token
of every row from them (temperature, top-k, top-p, min-p, from one given random
number a row), and `ebd_paged_plan` turns what the requests bring into page
tables, row positions and slots of the paged K/V cache, all on the device.

The sizes are this repository's own (the tiny, LLaDA-8B and Dream-7B widths and
vocabularies of `synth/configs.py`, windows of 1 to 64 rows, up to 64 sequences,
512 rows of a full sequence) and, beyond them, generic: odd vocabularies, rows
that are slices of wider buffers, thousands of sequences.  `draw` spreads over
the same ranges.

Logits: every row has a sharpness of its own, from nearly flat to one token that
has almost all, as the hidden rows of `synth/gen.py` do; some rows ban tokens
(-inf).  Every request brings its own sampling parameters.
"""
from __future__ import annotations

import math

import torch

own = False

# hidden size, vocabulary
TINY = (256, 4096)
LLADA_8B = (4096, 126464)
DREAM_7B = (3584, 152064)

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _logits(rows, d, vocab, pad=0, name=None):
    c = dict(entry="logits", rows=rows, d=d, vocab=vocab, pad=pad)
    return dict(c, name=name) if name else c


def _sample(rows, vocab, dtype, filters, pad=0, name=None):
    """filters: 'temperature', 'top_k', 'top_p', 'min_p', 'both' (top-k and
    top-p), 'greedy', or 'mixed': every row has its own."""
    c = dict(entry="sample", rows=rows, vocab=vocab, dtype=dtype, filters=filters, pad=pad)
    return dict(c, name=name) if name else c


def _plan(batch, add, length, page, ragged=False, name=None):
    c = dict(entry="plan", batch=batch, add=add, len=length, page=page, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest step: latency
        _logits(24, *TINY, name="logits_tiny"),
        # one user's window
        _logits(32, *LLADA_8B, name="logits_window"),
        # a batch's windows, into rows that leave room for added tokens
        _logits(390, *DREAM_7B, pad=57, name="logits_batch"),
        # one token at a temperature: latency
        _sample(1, TINY[1], "f32", "temperature", name="sample_one"),
        # one user's window, the usual settings
        _sample(32, LLADA_8B[1], "f32", "both", name="sample_window"),
        # one user's window by nucleus alone, of logits in 16 bits
        _sample(24, DREAM_7B[1], "bf16", "top_p", name="sample_nucleus"),
        # a batch at a temperature, nothing left out
        _sample(64, LLADA_8B[1], "f32", "temperature", name="sample_batch"),
        # an odd vocabulary, rows at odd addresses
        _sample(47, 57381, "f16", "min_p", pad=2, name="sample_odd"),
        # a server's batch: every request has its own settings
        _sample(512, DREAM_7B[1], "f32", "mixed", name="sample_requests"),
        # the next token of every sequence of a batch
        _plan(64, 1, 4096, 64, ragged=True, name="plan_tokens"),
        # prompts: many pages at once
        _plan(8, 512, 700, 16, ragged=True, name="plan_prompts"),
        # thousands of sequences with drafts of a token or two
        _plan(2048, 2, 2000, 16, ragged=True, name="plan_server"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


MAX_FLOPS = 2.0 * 390 * DREAM_7B[0] * DREAM_7B[1]  # logits_batch
MAX_LOGITS = 512 * DREAM_7B[1]                     # sample_requests


def draw(rng):
    entry = rng.choice(("logits", "sample", "sample", "sample", "plan"))
    if entry == "logits":
        d, vocab = rng.choice((TINY, LLADA_8B, DREAM_7B, (0, 0), (0, 0)))
        if d == 0:
            d, vocab = 8 * _log_int(rng, 8, 640), _log_int(rng, 1000, 160000)
        rows = _log_int(rng, 1, min(512, MAX_FLOPS / (2.0 * d * vocab)))
        return _logits(rows, d, vocab, pad=rng.choice((0, 0, 1, 64)))
    if entry == "sample":
        vocab = rng.choice((TINY[1], LLADA_8B[1], DREAM_7B[1], 0, 0, 0)) or _log_int(rng, 500, 200000)
        rows = _log_int(rng, 1, min(512, MAX_LOGITS / vocab))
        filters = rng.choice(("temperature", "top_k", "top_p", "min_p", "both", "mixed", "mixed", "greedy"))
        return _sample(rows, vocab, rng.choice(("f32", "f32", "bf16", "f16")), filters, pad=rng.choice((0, 0, 1, 8, 100)))
    batch = _log_int(rng, 1, 2048)
    add = _log_int(rng, 1, min(1024, 4096 // batch))
    return _plan(batch, add, _log_int(rng, 16, min(65536, 4200000 // batch)), rng.choice((16, 32, 64, 128)),
                 ragged=rng.random() < 0.7)


# ------------------------------------------------------------------ inputs
class _State:
    """What a program holds: weights or buffers, its handle, the call's inputs."""


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + what * 7919 + 29) % (1 << 62))


def _uniform(seed, what, shape, lo, hi):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(lo, hi, generator=_gen(seed, what))


def _normal(seed, what, shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=_gen(seed, what))


def prepare(case, seed):
    s = _State()
    s.case = case
    {"logits": _prepare_logits, "sample": _prepare_sample, "plan": _prepare_plan}[case["entry"]](s, case, seed)
    if own:
        _prepare_own(s, case)
    torch.cuda.synchronize()
    return s


def _prepare_logits(s, case, seed):
    rows, d, vocab = case["rows"], case["d"], case["vocab"]
    s.w = _normal(seed, 1, (vocab, d), torch.bfloat16).mul_(1.0 / math.sqrt(d))
    sharp = torch.exp(_uniform(seed, 2, (rows, 1), math.log(0.5), math.log(8.0)))
    s.h = (_normal(seed, 3, (rows, d)) * sharp).bfloat16()
    s.out = torch.zeros((rows, vocab + case["pad"]), dtype=torch.float32, device="cuda")[:, :vocab]


def _prepare_sample(s, case, seed):
    rows, vocab = case["rows"], case["vocab"]
    kind, dtype = case["filters"], TYPES[case["dtype"]]
    sharp = torch.exp(_uniform(seed, 1, (rows, 1), math.log(0.5), math.log(8.0)))
    buf = torch.zeros((rows, vocab + case["pad"]), dtype=dtype, device="cuda")
    s.logits = buf[:, :vocab]
    step = max(1, (1 << 26) // vocab)
    for i in range(0, rows, step):
        n = min(step, rows - i)
        x = _normal(seed, 100 + i, (n, vocab)) * sharp[i: i + n]
        banned = (_uniform(seed, 100000 + i, (n, vocab), 0, 1) < 0.01) & (_uniform(seed, 200000 + i, (n, 1), 0, 1) < 0.3)
        s.logits[i: i + n] = x.masked_fill(banned, -math.inf).to(dtype)
    s.u = _uniform(seed, 2, (rows,), 0, 1).clamp(max=1.0 - 2.0 ** -24)
    pick = _uniform(seed, 3, (rows,), 0, 1)
    every = kind == "mixed"

    def some(name, share):
        """Which rows have a filter."""
        if every:
            return _uniform(seed, 10 + len(name), (rows,), 0, 1) < share
        wanted = kind == name or (kind == "both" and name in ("top_k", "top_p"))
        return torch.full((rows,), wanted, dtype=torch.bool, device="cuda")

    s.temperature = torch.exp(_uniform(seed, 4, (rows,), math.log(0.3), math.log(1.5)))
    if every:
        s.temperature = torch.where(pick < 0.1, torch.zeros_like(s.temperature), s.temperature)
    if kind == "greedy":
        s.temperature = torch.zeros_like(s.temperature)
    s.top_k = s.top_p = s.min_p = None
    if every or kind in ("top_k", "both"):
        k = torch.exp(_uniform(seed, 5, (rows,), math.log(2.0), math.log(min(1000.0, vocab / 2)))).to(torch.int32)
        s.top_k = torch.where(some("top_k", 0.4), k, torch.zeros_like(k))
    if every or kind in ("top_p", "both"):
        p = _uniform(seed, 6, (rows,), 0.6, 0.99)
        s.top_p = torch.where(some("top_p", 0.5), p, torch.ones_like(p))
    if every or kind == "min_p":
        q = torch.exp(_uniform(seed, 7, (rows,), math.log(0.001), math.log(0.3)))
        s.min_p = torch.where(some("min_p", 0.2), q, torch.zeros_like(q))
    s.token = torch.zeros((rows,), dtype=torch.int32, device="cuda")
    s.prob = torch.zeros((rows,), dtype=torch.float32, device="cuda")


def _plan_lens(case):
    """Rows that every sequence brings, and its cached positions (host lists,
    part of the case)."""
    b, n, p = case["batch"], case["add"], case["len"]
    if not case["ragged"]:
        return [n] * b, [p] * b
    g = torch.Generator().manual_seed(b * 8191 + n * 131 + p)
    ns = torch.randint(0, n + 1, (b,), generator=g)
    if int(ns.sum()) == 0:
        ns[0] = n
    return ns.tolist(), torch.randint(0, p + 1, (b,), generator=g).tolist()


def _prepare_plan(s, case, seed):
    page, b = case["page"], case["batch"]
    ns, ps = _plan_lens(case)
    i32 = dict(dtype=torch.int32, device="cuda")
    held = [(p + page - 1) // page for p in ps]
    need = [(p + n + page - 1) // page for n, p in zip(ns, ps)]
    s.n_pages = sum(need) + 3
    # pages were handed out and given back in every order
    order = torch.randperm(s.n_pages, generator=torch.Generator().manual_seed(seed % (1 << 62))).to(torch.int32)
    width = max(max(need), 1)
    table = torch.full((b, width), -1, dtype=torch.int32)
    h = torch.tensor(held)
    used = int(h.sum())
    table[torch.arange(width)[None, :] < h[:, None]] = order[:used]
    s.table = table.cuda()
    s.free = torch.zeros((s.n_pages,), **i32)
    s.free[: s.n_pages - used] = order[used:].cuda()
    s.spare = s.n_pages - used
    s.n_free = torch.tensor([s.spare], **i32)
    s.kv_len = torch.tensor(ps, **i32)
    s.add = torch.tensor(ns, **i32)
    s.drop = -s.add
    s.rows = sum(ns)
    s.cu_rows = torch.zeros((b + 1,), **i32)
    s.row_pos = torch.zeros((s.rows,), **i32)
    s.slot = torch.zeros((s.rows,), dtype=torch.int64, device="cuda")


def _prepare_own(s, case):
    """The handle, the packed weights and the arguments that a program keeps."""
    from paper_2609_16450_gb300 import _ebd as E
    from paper_2609_16450_gb300 import runtime as rt
    s.E, s.rt = E, rt
    d, vocab = case.get("d", 64), case.get("vocab", 4096)
    rows = case["rows"] if "rows" in case else s.rows
    cfg = E.ebd_config(
        d_model=d, vocab=vocab, n_heads_q=4, n_heads_kv=4, head_dim=64, d_base=64,
        max_batch=case.get("batch", rows), max_window=1 if case["entry"] == "plan" else min(64, rows),
        max_rows=rows, max_prefix=0, gen_len=64, g_max=5, l_min=8, l_b=32, eos_id=vocab - 1, lps_enabled=1,
        tau=0.9, tau_psi=0.89, paged=0 if case["entry"] == "logits" else 1)
    s.handle = rt.Handle(cfg)
    if case["entry"] == "logits":
        w = rt.pack_weights(s.handle, rt.DeviceWeights(w_lm=s.w, w_emb=None))
        s.w = w.w_lm
        a = s.args = E.ebd_step_args()
        a.batch, a.rows = rows, rows
        a.hidden, a.w_lm, a.w_lm_layout = s.h.data_ptr(), w.w_lm.data_ptr(), w.layout
        return
    if case["entry"] == "sample":
        a = s.args = E.ebd_sample_args()
        a.rows, a.dtype = rows, {"f32": E.EBD_LOGITS_F32, "bf16": E.EBD_LOGITS_BF16, "f16": E.EBD_LOGITS_F16}[case["dtype"]]
        a.logits, a.stride, a.u = s.logits.data_ptr(), s.logits.stride(0), s.u.data_ptr()
        for name in ("temperature", "top_k", "top_p", "min_p"):
            setattr(a, name, rt.ptr(getattr(s, name)))
        a.token, a.prob = s.token.data_ptr(), s.prob.data_ptr()
        return

    def plan(add, out):
        a = E.ebd_paged_plan_args()
        a.batch, a.rows = case["batch"], s.rows if out else 0
        a.add, a.kv_len, a.page_table = add.data_ptr(), s.kv_len.data_ptr(), s.table.data_ptr()
        a.free_pages, a.n_free = s.free.data_ptr(), s.n_free.data_ptr()
        if out:
            a.cu_rows, a.row_pos, a.slot = s.cu_rows.data_ptr(), s.row_pos.data_ptr(), s.slot.data_ptr()
        a.page_size, a.n_pages, a.max_pages = case["page"], s.n_pages, s.table.shape[1]
        return a

    s.grow, s.shrink = plan(s.add, True), plan(s.drop, False)


# ------------------------------------------------------------------ one pass
def run(s):
    if s.case["entry"] == "logits":
        if own:
            s.E.check(s.E.ebd_lm_logits(s.handle.h, s.args, s.out.data_ptr(), s.out.stride(0), s.rt.stream_handle(None)),
                      s.handle.h)
        else:
            s.out = s.h.float() @ s.w.float().T
        return s.out
    if s.case["entry"] == "sample":
        if own:
            s.E.check(s.E.ebd_sample(s.handle.h, s.args, s.rt.stream_handle(None)), s.handle.h)
        else:
            _plain_sample(s)
        return {"token": s.token, "prob": s.prob}
    # A step reserves its rows, and what was not accepted (here: none was) goes
    # back: the lengths and the order of the free pages are then as before.
    if own:
        stream = s.rt.stream_handle(None)
        s.E.check(s.E.ebd_paged_plan(s.handle.h, s.grow, stream), s.handle.h)
        s.E.check(s.E.ebd_paged_plan(s.handle.h, s.shrink, stream), s.handle.h)
    else:
        _plain_plan(s, s.add, True)
        _plain_plan(s, s.drop, False)
    return {"cu_rows": s.cu_rows, "row_pos": s.row_pos, "slot": s.slot, "kv_len": s.kv_len, "table": s.table,
            "free": s.free[: s.spare], "n_free": s.n_free}


def _plain_sample(s):
    """In 64 bits: a token's border in the sum of all is 1e-6 of it away from the
    next one's, and has to be on the right side of u."""
    rows = s.logits.shape[0]
    step = max(1, (1 << 25) // s.logits.shape[1])
    out = [_plain_rows(s, slice(i, min(rows, i + step))) for i in range(0, rows, step)]
    s.token, s.prob = (torch.cat(t) for t in zip(*out))


def _plain_rows(s, at):
    l = s.logits[at].double()
    n, vocab = l.shape
    temp = s.temperature[at].double()[:, None]
    greedy = temp == 0
    x = (l - l.amax(-1, keepdim=True)) / torch.where(greedy, torch.ones_like(temp), temp)
    w = torch.exp(x)
    w = torch.where(x >= -40 * math.log(2.0), w, torch.zeros_like(w))
    # by descending logit, the lower index first
    order = torch.sort(l, dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    rank = torch.arange(vocab, device=l.device)[None, :]
    kept = torch.ones_like(l, dtype=torch.bool)
    if s.top_k is not None:
        k = s.top_k[at].long()[:, None]
        kept &= (rank < k) | (k <= 0)
    if s.top_p is not None:
        p = s.top_p[at].double()[:, None]
        wk = torch.where(kept, ws, torch.zeros_like(ws))
        before = wk.cumsum(-1)
        total = before[:, -1:]
        before = torch.cat((torch.zeros_like(total), before[:, :-1]), 1)
        kept &= (before < p * total) | (p >= 1) | (rank == 0)
    if s.min_p is not None:
        kept &= x.gather(1, order) >= torch.log(s.min_p[at].double())[:, None]
    kept &= (rank == 0) | ~greedy
    w = torch.where(torch.zeros_like(kept).scatter(1, order, kept), w, torch.zeros_like(w))
    upto = w.cumsum(-1)
    total = upto[:, -1:]
    token = torch.searchsorted(upto, s.u[at].double()[:, None] * total, right=True)
    return token[:, 0].to(torch.int32), (w.gather(1, token) / total)[:, 0].float()


def _plain_plan(s, add, out):
    page, width = s.case["page"], s.table.shape[1]
    old = s.kv_len.long()
    new = (old + add.long()).clamp(min=0)
    have, want = (old + page - 1) // page, (new + page - 1) // page
    j = torch.arange(width, device="cuda")
    # back: sequences from the last to the first, their last page first
    gone = ((j >= want[:, None]) & (j < have[:, None])).flatten()
    n = s.n_free.long()
    back = gone.long().flip(0).cumsum(0).flip(0)
    stack = torch.cat((s.free, s.free.new_zeros(1)))
    at = torch.where(gone, n + back - 1, torch.full_like(back, s.n_pages))
    stack.scatter_(0, at, s.table.flatten())
    n = n + gone.sum()
    table = s.table.flatten().masked_fill(gone, -1)
    # out: sequences and pages ascending, from the top
    more = ((j >= have[:, None]) & (j < want[:, None])).flatten()
    rank = more.long().cumsum(0)
    table = torch.where(more, stack[(n - rank).clamp(min=0)], table)
    s.table = table.view_as(s.table)
    s.free, s.n_free, s.kv_len = stack[:-1].clone(), (n - more.sum()).to(torch.int32), new.to(torch.int32)
    if not out:
        return
    cu = torch.cat((old.new_zeros(1), add.long().clamp(min=0).cumsum(0)))
    r = torch.arange(s.rows, device="cuda")
    b = torch.searchsorted(cu[1:], r, right=True)
    pos = old[b] + r - cu[b]
    s.cu_rows, s.row_pos = cu.to(torch.int32), pos.to(torch.int32)
    s.slot = s.table[b, pos // page].long() * page + pos % page


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["entry"] == "logits":
        rows, d, vocab = case["rows"], case["d"], case["vocab"]
        return {"bytes": 2.0 * (vocab + rows) * d + 4.0 * rows * vocab, "flops": 2.0 * rows * vocab * d}
    if case["entry"] == "sample":
        n = float(case["rows"]) * case["vocab"]
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + 28.0 * case["rows"], "flops": 4.0 * n}
    ns, ps = _plan_lens(case)
    page = case["page"]
    moved = sum((p + n + page - 1) // page - (p + page - 1) // page for n, p in zip(ns, ps))
    # both calls: lengths and their changes; pages from the stack into the table
    # and back; the rows' positions and slots
    return {"bytes": 2.0 * 12 * case["batch"] + 2.0 * 8 * moved + 12.0 * sum(ns) + 4.0, "flops": 8.0 * sum(ns)}


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    return {"logits": _exact_logits, "sample": _exact_sample, "plan": _exact_plan}[case["entry"]](case, seed)


def _fresh(case, seed):
    """The inputs without the framework's part."""
    s = _State()
    s.case = case
    {"logits": _prepare_logits, "sample": _prepare_sample, "plan": _prepare_plan}[case["entry"]](s, case, seed)
    return s


def _exact_logits(case, seed):
    s = _fresh(case, seed)
    out = torch.empty((case["rows"], case["vocab"]), dtype=torch.float64, device="cuda")
    h = s.h.double()
    for i in range(0, case["vocab"], 8192):
        out[:, i: i + 8192] = torch.mm(h, s.w[i: i + 8192].double().t())
    return out


def _exact_sample(case, seed):
    """Row by row: a threshold on the logit and the index, then the sum up to u."""
    s = _fresh(case, seed)
    tokens, probs = [], []
    for r in range(case["rows"]):
        l = s.logits[r].double()
        t = float(s.temperature[r])
        if t == 0:
            tokens.append(int((l == l.max()).nonzero()[0]))
            probs.append(1.0)
            continue
        x = (l - l.max()) / t
        w = torch.where(x < -40 * math.log(2.0), 0.0, torch.exp(x))
        idx = torch.argsort(-l, stable=True)
        if s.top_k is not None and int(s.top_k[r]) > 0:
            idx = idx[: int(s.top_k[r])]
        if s.top_p is not None and float(s.top_p[r]) < 1:
            c = torch.cumsum(w[idx], 0)
            idx = idx[: int((c < float(s.top_p[r]) * c[-1]).sum()) + 1]
        if s.min_p is not None and float(s.min_p[r]) > 0:
            idx = idx[x[idx] >= math.log(float(s.min_p[r]))]
        idx = torch.sort(idx).values
        c = torch.cumsum(w[idx], 0)
        i = int((c <= float(s.u[r]) * c[-1]).sum())
        tokens.append(int(idx[i]))
        probs.append(float(w[idx[i]] / c[-1]))
    return {"token": torch.tensor(tokens, dtype=torch.int32, device="cuda"),
            "prob": torch.tensor(probs, dtype=torch.float64, device="cuda")}


def _exact_plan(case, seed):
    s = _fresh(case, seed)
    page = case["page"]
    free = s.free.tolist()[: int(s.n_free)]
    first, table, lens = list(free), s.table.tolist(), s.kv_len.tolist()
    cu, pos, slot = [0], [], []
    for b, n in enumerate(s.add.tolist()):
        have = -(-lens[b] // page)
        for i in range(have, -(-(lens[b] + n) // page)):
            table[b][i] = free.pop()
        for p in range(lens[b], lens[b] + n):
            pos.append(p)
            slot.append(table[b][p // page] * page + p % page)
        cu.append(len(pos))
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"cu_rows": torch.tensor(cu, **i32), "row_pos": torch.tensor(pos, **i32),
            "slot": torch.tensor(slot, dtype=torch.int64, device="cuda"), "kv_len": s.kv_len, "table": s.table,
            "free": torch.tensor(first, **i32), "n_free": s.n_free}
