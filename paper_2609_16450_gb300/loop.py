"""Host driver of the generation loop (App. E algorithm, in the block-forward
window setting of Sec. 6.4) for one sequence: a committed prompt of
`prefix` positions followed by `gen_len` masked response positions.

Each step asks the library for the next window (ebd_loop_window), has the
caller supply that window's backbone outputs (hidden states, q, k, v) and
runs ebd_step on it.  The decode state (tokens, mask, block flags, block
meta) of the whole response stays on the device; a step's window is a slice
of it.  The K/V cache is indexed by absolute position; a step attends to its
first prefix + frontier rows (prefix cache) and, with cache='dual', also to
the positions right of the window (dual cache, Sec. 6.3).  With append=True
each step writes the K/V of the rows it commits into the cache
(ebd_step_args.kv_append); the cache then starts with the prompt only.
With cache='paged' the K/V live in a PagedCache: the prompt's rows are written
into it piece by piece, every step writes its window's rows into pages reserved
as the window moves on (ebd_paged_write) and attends to all positions up to the
window's end (ebd_paged_attention), and the cache is read back at the end
(ebd_paged_read).
With plan='device' those pages are handed out by ebd_paged_plan: what the last window
cached past the new window's start goes back, and the window's rows come.
With `sampling` x_hat is drawn at a temperature (ebd_lm_logits, ebd_sample) and kappa is
the probability it was drawn with; the decision then runs on them (ebd_decide).  Where one
token is left to draw (temperature 0, top_k 1, a top_p near 0) that is 1, and the decision
accepts every row that it looks at (top-m, the first m of them): argmax decoding, with kappa =
max p, is the loop without `sampling`.
This module only marshals buffers; the window rule and every step of the
method run in the library."""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import Callable, List, Optional

import numpy as np
import torch

from . import _ebd as E
from . import runtime as rt
from . import sampling as sp
from .paged import PagedCache

MASK_TOKEN = -1


@dataclass
class LoopStep:
    step: int
    window: tuple
    accepted: np.ndarray
    argmax: np.ndarray
    conf: np.ndarray
    lbs_logit: np.ndarray
    lps_prob: np.ndarray
    attn_out: Optional[np.ndarray]
    device_us: float
    # the window's statistics and decode state before and after the step
    entropy: Optional[np.ndarray] = None
    ent_norm: Optional[np.ndarray] = None
    gap: Optional[np.ndarray] = None
    before: Optional[dict] = None
    after: Optional[dict] = None


@dataclass
class LoopResult:
    tokens: np.ndarray
    steps: int
    commits: List[int] = field(default_factory=list)
    records: List[LoopStep] = field(default_factory=list)
    device_us: float = 0.0
    k_cache: Optional[np.ndarray] = None  # [P0 + L][Hkv][D] int16 bits after the loop
    v_cache: Optional[np.ndarray] = None


def config_for_loop(shape, max_window: int = 64, decode_mode: int = E.EBD_DECODE_EB,
                    top_m: int = 1, paged: int = 0) -> E.ebd_config:
    return rt.config_for(shape, max_batch=1, max_window=max_window, max_rows=max_window,
                         max_prefix=shape.prefix + shape.gen_len, decode_mode=decode_mode,
                         top_m=top_m, paged=paged)


def run_loop(h: rt.Handle, shape, weights: rt.DeviceWeights,
             window_inputs: Callable, kv_rows: Callable, attention: bool = True,
             max_steps: Optional[int] = None, max_window: int = 64,
             keep: bool = True, stream: Optional[torch.cuda.Stream] = None,
             block: int = 32, cache: str = "prefix", append: bool = False,
             window: str = "block", page_size: int = 64, kv_dtype: str = "bf16", plan: str = "host",
             sampling: Optional[sp.Settings] = None, uniforms: Optional[Callable] = None) -> LoopResult:
    """window_inputs(step, positions) -> (hidden, q, k_win, v_win) as bf16 bit
    arrays; kv_rows(positions) -> (k, v).  Positions are absolute.  Under the
    handle's baseline decode modes the window is the active fixed block of
    `block` positions (ebd_loop_block_window).  cache: 'prefix' or 'dual';
    append: the step appends committed rows' K/V to the cache, which starts
    with the prompt's K/V only (with 'dual', with every position's, the
    positions right of the window standing for the K/V a dual cache holds).
    cache='paged' (a handle of ebd_config.paged = 1): pages of page_size
    positions in kv_dtype, 'bf16' or 'e4m3', planned on the 'host' or the 'device'; the
    attention's outputs are bf16.  sampling: how x_hat is drawn, by uniforms(step,
    positions) -> one number in [0, 1) per position; a step then does not append."""
    if cache not in ("prefix", "dual", "paged"):
        raise ValueError("cache must be 'prefix', 'dual' or 'paged'")
    paged = cache == "paged"
    if paged and append:
        raise ValueError("the paged cache takes every window's rows: it has no append")
    if window not in ("block", "full"):
        raise ValueError("window must be 'block' or 'full'")
    if plan not in ("host", "device") or (plan == "device" and not paged):
        raise ValueError("plan must be 'host', or 'device' with the paged cache")
    if sampling is not None and (append or uniforms is None):
        raise ValueError("sampling needs uniforms, and appends nothing")
    full = window == "full"  # the full-sequence setting: the window is the whole response
    if full and (attention or append or paged):
        raise ValueError("the full-sequence window runs without the window attention")
    fixed = h.cfg.decode_mode != E.EBD_DECODE_EB
    dev = "cuda"
    P0, L = shape.prefix, shape.gen_len
    d, Hq, Hkv, D = shape.d_model, shape.n_heads_q, shape.n_heads_kv, shape.head_dim
    W = L if full else max_window
    stream = stream or torch.cuda.current_stream()
    sid = stream.cuda_stream
    i32 = dict(dtype=torch.int32, device=dev)
    u8 = dict(dtype=torch.uint8, device=dev)
    f32 = dict(dtype=torch.float32, device=dev)
    tokens = torch.full((L,), MASK_TOKEN, **i32)
    mask = torch.ones((L,), **u8)
    in_block = torch.zeros((L,), **u8)
    meta = torch.zeros((2,), **i32)
    mask_h = np.ones(L, np.uint8)
    ib_h = np.zeros(L, np.uint8)
    meta_h = np.zeros(2, np.int32)
    # window inputs, outputs and the K/V of every position
    hid = torch.empty((W, d), dtype=torch.int16, device=dev)
    q = torch.empty((W, Hq, D), dtype=torch.int16, device=dev)
    kw = torch.empty((W, Hkv, D), dtype=torch.int16, device=dev)
    vw = torch.empty((W, Hkv, D), dtype=torch.int16, device=dev)
    cu = torch.zeros((2,), **i32)
    pl = torch.zeros((1,), **i32)
    rp = torch.zeros((W,), **i32)
    outs = {k: torch.empty((W,), **f32) for k in ("conf", "entropy", "ent_norm", "gap",
                                                  "lbs_logit", "lps_prob")}
    argmax = torch.empty((W,), **i32)
    accepted = torch.empty((W,), **u8)
    attn_out = torch.empty((W, Hq, D), **f32) if attention else None
    kc = vc = None
    sfx = torch.zeros((2,), **i32)
    dense = not paged and (attention or append)
    if dense:
        n0 = P0 if (append and cache == "prefix") else P0 + L
        kk, vv = kv_rows(np.arange(n0, dtype=np.int32))
        kc = torch.zeros((1, P0 + L, Hkv, D), dtype=torch.int16, device=dev)
        vc = torch.zeros((1, P0 + L, Hkv, D), dtype=torch.int16, device=dev)
        kc[0, :n0] = rt._dev(kk, dev).reshape(n0, Hkv, D)
        vc[0, :n0] = rt._dev(vv, dev).reshape(n0, Hkv, D)
    if paged:
        n_pages = (P0 + L + page_size - 1) // page_size
        device_plan = plan == "device"
        kv_len = torch.zeros((1,), **i32)
        add = torch.zeros((1,), **i32)
        cached = 0  # positions that the plan has
        attn_p = torch.empty((W, Hq, D), dtype=torch.bfloat16, device=dev)
        with torch.cuda.stream(stream):
            pages = PagedCache(h, n_pages, 1, n_pages, page_size, kv_dtype, plan=plan)
            if device_plan:
                kv_len = pages.kv_len
            else:
                pages.reserve(0, P0, stream)
            for at in range(0, P0, W):  # the prompt, in pieces that the handle's rows hold
                pos = np.arange(at, min(at + W, P0), dtype=np.int32)
                kk, vv = kv_rows(pos)
                if device_plan:
                    add.copy_(torch.tensor([len(pos)], dtype=torch.int32))
                    pages.plan(add, cu, rp, stream=stream)
                    at_cu, at_pos = cu, rp[:len(pos)]
                else:
                    at_cu, at_pos = rt._dev(np.array([0, len(pos)], np.int32), dev), rt._dev(pos, dev)
                pages.write(at_cu, at_pos, rt._dev(kk, dev).view(-1, Hkv, D), rt._dev(vv, dev).view(-1, Hkv, D),
                            stream=stream)
            cached = P0
    if sampling is not None:
        logits = torch.empty((W, shape.vocab), **f32)
        u = torch.empty((W,), **f32)
        drawn = sampling.rows(W, dev)
    ev0, ev1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    res = LoopResult(tokens=None, steps=0)
    step = 0
    while True:
        if max_steps is not None and step >= max_steps:
            break
        if full:
            s, lo, hi = E.EBD_OK, (0 if mask_h.any() else L), L
        elif fixed:
            s, lo, hi = E.ebd_loop_block_window(mask_h, block)
        else:
            s, lo, hi = E.ebd_loop_window(mask_h, ib_h, meta_h, W)
        if s != E.EBD_OK:
            raise E.EbdError(s, "loop window")
        if lo >= L:
            break
        R = hi - lo
        positions = (P0 + np.arange(lo, hi)).astype(np.int32)
        h_b, q_b, k_b, v_b = window_inputs(step, positions)
        with torch.cuda.stream(stream):
            hid[:R].copy_(torch.from_numpy(np.ascontiguousarray(h_b).view(np.int16)).reshape(R, d))
            q[:R].copy_(torch.from_numpy(np.ascontiguousarray(q_b).view(np.int16)).reshape(R, Hq, D))
            kw[:R].copy_(torch.from_numpy(np.ascontiguousarray(k_b).view(np.int16)).reshape(R, Hkv, D))
            vw[:R].copy_(torch.from_numpy(np.ascontiguousarray(v_b).view(np.int16)).reshape(R, Hkv, D))
            cu.copy_(torch.tensor([0, R], dtype=torch.int32))
            pl.copy_(torch.tensor([P0 + lo], dtype=torch.int32))
            rp[:R].copy_(torch.from_numpy(positions))
            sfx.copy_(torch.tensor([P0 + hi, L - hi], dtype=torch.int32))
            if paged and device_plan:
                add.copy_(torch.tensor([P0 + lo - cached], dtype=torch.int32))
                if cached > P0 + lo:
                    pages.plan(add, stream=stream)
                    cached = P0 + lo
                add.copy_(torch.tensor([P0 + hi - cached], dtype=torch.int32))
                pages.plan(add, cu, rp, stream=stream)
                cached = P0 + hi
            elif paged:
                kv_len.copy_(torch.tensor([P0 + hi], dtype=torch.int32))
                pages.reserve(0, P0 + hi, stream)
            if sampling is not None:
                u[:R].copy_(torch.from_numpy(np.ascontiguousarray(uniforms(step, positions), dtype=np.float32)))
        a = E.ebd_step_args()
        a.batch, a.rows = 1, R
        a.cu_rows, a.prefix_len, a.row_pos = cu.data_ptr(), pl.data_ptr(), rp.data_ptr()
        a.hidden, a.q, a.k_win, a.v_win = hid.data_ptr(), q.data_ptr(), kw.data_ptr(), vw.data_ptr()
        if dense:
            a.k_cache, a.v_cache = kc.data_ptr(), vc.data_ptr()
        if attention and not paged:
            a.attn_out = attn_out.data_ptr()
            if cache == "dual":
                a.suffix = sfx.data_ptr()
        a.kv_append = 1 if append else 0
        a.w_lm, a.w_lm_layout = weights.w_lm.data_ptr(), weights.layout
        a.tokens = tokens.data_ptr() + 4 * lo
        a.mask = mask.data_ptr() + lo
        a.in_block = in_block.data_ptr() + lo
        a.blk_meta = meta.data_ptr()
        for k, t in outs.items():
            setattr(a, k, t.data_ptr())
        a.argmax, a.accepted = argmax.data_ptr(), accepted.data_ptr()
        before = int(mask_h.sum())
        if keep:
            snap = dict(tokens=tokens[lo:hi].cpu().numpy(), mask=mask_h[lo:hi].copy(),
                        in_block=ib_h[lo:hi].copy(), meta=meta_h.copy())
        ev0.record(stream)
        if paged:
            pages.write(cu, rp[:R], kw[:R], vw[:R], stream=stream)
            if attention:
                pages.attention(q[:R], cu, kv_len, attn_p[:R], stream=stream)
        if sampling is None:
            E.check(E.ebd_step(h.h, a, sid), h.h)
        else:
            with torch.cuda.stream(stream):
                sp.lm_logits(h, hid[:R], weights, logits[:R],
                             {k: outs[k][:R] for k in ("entropy", "ent_norm", "gap")}, stream)
                sp.sample(h, logits[:R], u[:R], argmax[:R], outs["conf"][:R], stream=stream,
                          **{k: None if t is None else t[:R] for k, t in drawn.items()})
            if attention and not paged:
                E.check(E.ebd_attention(h.h, a, sid), h.h)
            E.check(E.ebd_decide(h.h, a, sid), h.h)
        ev1.record(stream)
        st = h.sync_status(stream)
        if st != 0:
            raise E.EbdError(st, E.ebd_last_error(h.h))
        us = ev0.elapsed_time(ev1) * 1000.0
        mask_h = mask.cpu().numpy()
        ib_h = in_block.cpu().numpy()
        meta_h = meta.cpu().numpy()
        if keep:
            after = dict(tokens=tokens[lo:hi].cpu().numpy(), mask=mask_h[lo:hi].copy(),
                         in_block=ib_h[lo:hi].copy(), meta=meta_h.copy())
        if meta_h[1] == 0 and ib_h.any():
            # a resolved block releases its flags outside the window too
            in_block.zero_()
            ib_h[:] = 0
        res.commits.append(before - int(mask_h.sum()))
        res.device_us += us
        if keep:
            res.records.append(LoopStep(
                step=step, window=(lo, hi), accepted=accepted[:R].cpu().numpy(),
                argmax=argmax[:R].cpu().numpy(), conf=outs["conf"][:R].cpu().numpy(),
                lbs_logit=outs["lbs_logit"][:R].cpu().numpy(),
                lps_prob=outs["lps_prob"][:R].cpu().numpy(),
                attn_out=((attn_p if paged else attn_out)[:R].float().cpu().numpy()
                          if attention else None), device_us=us,
                entropy=outs["entropy"][:R].cpu().numpy(), ent_norm=outs["ent_norm"][:R].cpu().numpy(),
                gap=outs["gap"][:R].cpu().numpy(), before=snap, after=after))
        step += 1
    res.tokens = tokens.cpu().numpy()
    res.steps = step
    if paged:
        n = P0 + L
        with torch.cuda.stream(stream):
            kc, vc = (torch.empty((1, n, Hkv, D), dtype=torch.int16, device=dev) for _ in range(2))
            for at in range(0, n, W):
                pos = np.arange(at, min(at + W, n), dtype=np.int32)
                pages.read(rt._dev(np.array([0, len(pos)], np.int32), dev), rt._dev(pos, dev),
                           kc[0, at: at + W], vc[0, at: at + W], stream=stream)
        st = h.sync_status(stream)
        if st != 0:
            raise E.EbdError(st, E.ebd_last_error(h.h))
    if kc is not None:
        res.k_cache, res.v_cache = kc[0].cpu().numpy(), vc[0].cpu().numpy()
    return res
