"""Draws under temperature, top-k, top-p and min-p, and rows truncated the same way (see spec_sample_rows in include/spec.h).

Argument marshalling only.  Every call runs on the current stream of the logits' device.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import Sampling, load_library
from .binding import call_on, need


def _sampling(temperature: float, logit_scale: float, top_k: int, top_p: float, min_p: float) -> Sampling:
    need(0 <= top_k < 1 << 31, "top_k: 0 or a number of ids")            # the struct would keep its low 32 bits
    return Sampling(temperature, logit_scale, top_k, top_p, min_p)


def _call(logits: torch.Tensor, u, sampling, want_q: bool, masked, want_tokens: bool):
    if not (logits.is_cuda and logits.dtype is torch.float32 and logits.dim() == 2 and
            (logits.stride(1) == 1 or logits.shape[1] == 1)):
        raise ValueError("logits: rows in float32 on a GPU are wanted")
    n, V = logits.shape
    if n >> 31 or V >> 31:                                               # ctypes would keep the low 32 bits
        raise ValueError("logits: too many rows or ids")
    lib = load_library()
    work = logits.new_empty(lib.spec_sample_rows_workspace_bytes(n, V) or 16, dtype=torch.uint8)
    q = logits.new_empty((n, V)) if want_q else None
    tokens = logits.new_empty(n, dtype=torch.int32) if want_tokens else None
    call_on(logits.get_device(), lib.spec_sample_rows, logits.data_ptr(), logits.stride(0) if n > 1 else V, n, V,
            C.byref(sampling), u.data_ptr() if u is not None else None, q.data_ptr() if want_q else None,
            masked.data_ptr() if masked is not None else None, tokens.data_ptr() if want_tokens else None, work.data_ptr())
    return tokens, q


def sample_rows(logits: torch.Tensor, u: Optional[torch.Tensor], temperature: float = 1.0, logit_scale: float = 1.0,
                top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0,
                want_q: bool = True) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """A token per row of fp32 logits [n][vocab] (any row stride) by the uniforms u [n] (fp32, on the GPU; None at temperature
    0): (tokens int32 [n], the distributions they were drawn from [n][vocab], or None if not wanted)."""
    if u is not None:
        if not (u.dtype is torch.float32 and u.is_contiguous() and u.get_device() == logits.get_device() and
                u.numel() == logits.shape[0]):
            raise ValueError("u: float32 [n] on the device of the logits is wanted")
    return _call(logits, u, _sampling(temperature, logit_scale, top_k, top_p, min_p), want_q, None, True)


def filter_rows(logits: torch.Tensor, temperature: float = 1.0, logit_scale: float = 1.0, top_k: int = 0, top_p: float = 1.0,
                min_p: float = 0.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The logits with -inf where sample_rows would keep no id: p_logits for accept_rows with the same temperature and
    logit_scale.  out: contiguous [n][vocab], may be the logits, but not overlap them otherwise."""
    if out is None:
        out = torch.empty(logits.shape, dtype=torch.float32, device=logits.device)
    need(out.dtype == torch.float32 and out.is_contiguous() and out.device == logits.device and out.shape == logits.shape,
         "out: contiguous float32 of the logits' shape is wanted")
    _call(logits, None, _sampling(temperature, logit_scale, top_k, top_p, min_p), False, out, False)
    return out
