"""Decoding at a temperature: the logits of a step's rows in memory (ebd_lm_logits) and
tokens drawn from them (ebd_sample), on torch tensors.  What is drawn goes into
ebd_decide as argmax and conf; a token that was the only one to draw (temperature 0) has
conf 1, for which lm_logits' conf may stand in.

    lm_logits(h, hidden, weights, logits, stats={"entropy": ent, "ent_norm": hn, "gap": gap})
    sample(h, logits, u, token, prob, temperature=t, top_k=k, top_p=p)

These functions check and marshal; every computation is a kernel of libebd.so.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, Optional

import torch

from . import _ebd as E
from . import runtime as rt

DTYPES = {torch.float32: E.EBD_LOGITS_F32, torch.bfloat16: E.EBD_LOGITS_BF16, torch.float16: E.EBD_LOGITS_F16}
STATS = {"conf": torch.float32, "entropy": torch.float32, "ent_norm": torch.float32, "gap": torch.float32,
         "argmax": torch.int32}


@dataclass
class Settings:
    """One setting for all rows; ebd_sample_args has what they mean."""
    temperature: float = 1.0
    top_k: int = 0
    top_p: float = 1.0
    min_p: float = 0.0

    def rows(self, n: int, device="cuda") -> Dict[str, Optional[torch.Tensor]]:
        """What sample() takes for n rows; filters that are off are left out (NaN is not off:
        rows that have it are refused)."""
        f32 = dict(dtype=torch.float32, device=device)
        return dict(
            temperature=torch.full((n,), self.temperature, **f32),
            top_k=torch.full((n,), self.top_k, dtype=torch.int32, device=device) if self.top_k > 0 else None,
            top_p=torch.full((n,), self.top_p, **f32) if not self.top_p >= 1 else None,
            min_p=torch.full((n,), self.min_p, **f32) if not self.min_p <= 0 else None)


def _matrix(t: torch.Tensor, what: str, width: int) -> int:
    """Stride between the rows of a [rows][width] tensor, which may be a slice."""
    if t.dim() != 2 or t.shape[1] != width:
        raise ValueError(f"{what}: [rows][{width}] expected, not {list(t.shape)}")
    if t.shape[0] and t.stride(1) != 1:
        raise ValueError(f"{what}: a row must be contiguous")
    if t.shape[0] < 2:
        return 0
    if t.stride(0) < width:  # an expanded row among them: a stride of 0 is dense to the C calls
        raise ValueError(f"{what}: rows must not overlap (stride {t.stride(0)} of rows of {width})")
    return t.stride(0)


def _vector(t: torch.Tensor, what: str, rows: int, dtype, device) -> int:
    if t.dtype != dtype or t.shape != (rows,) or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {dtype} [{rows}] expected, not {t.dtype} {list(t.shape)}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, not on {device}")
    return t.data_ptr()


def lm_logits(h: rt.Handle, hidden: torch.Tensor, weights: rt.DeviceWeights, logits: torch.Tensor,
              stats: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> None:
    """logits [rows][vocab] fp32 (rows of a wider buffer too) = hidden [rows][d_model]
    bf16 (or its bits) times W_lm; `stats`: vectors of `STATS` to be filled beside them."""
    c = h.cfg
    if hidden.dtype not in (torch.bfloat16, torch.int16) or hidden.dim() != 2 or hidden.shape[1] != c.d_model:
        raise ValueError(f"hidden: bf16 [rows][{c.d_model}] expected, not {hidden.dtype} {list(hidden.shape)}")
    if not hidden.is_contiguous():
        raise ValueError("hidden: contiguous rows expected")
    rows = hidden.shape[0]
    if logits.dtype != torch.float32 or logits.shape[:1] != (rows,):
        raise ValueError(f"logits: fp32 [{rows}][{c.vocab}] expected, not {logits.dtype} {list(logits.shape)}")
    stride = _matrix(logits, "logits", c.vocab)
    for what, t in (("logits", logits), ("W_lm", weights.w_lm)):
        if t.device != hidden.device:
            raise ValueError(f"{what} is on {t.device}, hidden on {hidden.device}")
    rt.check_device(h, "hidden", hidden)
    a = E.ebd_step_args()
    # the LM head takes rows as they come: any sequences that hold them
    a.batch, a.rows = c.max_batch, rows
    a.hidden, a.w_lm, a.w_lm_layout = hidden.data_ptr(), weights.w_lm.data_ptr(), weights.layout
    for name, t in (stats or {}).items():
        if name not in STATS:
            raise ValueError(f"no statistic {name!r}")
        setattr(a, name, _vector(t, name, rows, STATS[name], hidden.device))
    E.check(E.ebd_lm_logits(h.h, a, logits.data_ptr(), stride, rt.stream_handle(stream)), h.h)


def sample(h: rt.Handle, logits: torch.Tensor, u: torch.Tensor, token: torch.Tensor, prob: torch.Tensor,
           temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
           top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, stream=None) -> None:
    """token [rows] int32 and prob [rows] fp32 drawn from logits [rows][vocab] (fp32, bf16
    or fp16, rows of a wider buffer too) by u [rows] in [0, 1), each row by its own
    temperature, top-k, top-p and min-p."""
    if logits.dtype not in DTYPES:
        raise ValueError(f"logits: fp32, bf16 or fp16 expected, not {logits.dtype}")
    stride = _matrix(logits, "logits", h.cfg.vocab)
    rows, dev = logits.shape[0], logits.device
    rt.check_device(h, "logits", logits)
    a = E.ebd_sample_args()
    a.rows, a.dtype, a.logits, a.stride = rows, DTYPES[logits.dtype], logits.data_ptr(), stride
    for name, t, dtype in (("u", u, torch.float32), ("token", token, torch.int32), ("prob", prob, torch.float32),
                           ("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                           ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if t is not None:
            setattr(a, name, _vector(t, name, rows, dtype, dev))
    E.check(E.ebd_sample(h.h, a, rt.stream_handle(stream)), h.h)
