"""Verification of drafted tokens (``pipo_op_verify_drafts`` of ``include/pipo.h``) on
torch tensors.

The drafts of sequence b are entries ``start[b] .. start[b+1]-1`` of ``drafted``; the target's
probabilities have one row for each of them and one for the token behind the last,
in order: row ``start[b] + b + i`` belongs to draft i of sequence b.  Random
numbers are the caller's.  The call runs on the current CUDA stream of the tensors' device,
reads ``start`` there and does not synchronise.  There is no backward pass.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import capi

_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice
_TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _rows(x: torch.Tensor, n: int, vocab: int, dtype: torch.dtype, device: torch.device, name: str) -> int:
    """Row stride of probabilities [n, vocab]."""
    if x.shape != (n, vocab) or x.dtype is not dtype or x.device != device or (n and vocab > 1 and x.stride(1) != 1):
        raise ValueError(f"{name} must be [{n}, {vocab}] {dtype} with whole rows on {device}")
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and the verification has none")
    return x.stride(0) if n > 1 else vocab


def verify(target: torch.Tensor, drafted: torch.Tensor, start: torch.Tensor, u: torch.Tensor, r: torch.Tensor, *,
           width: int, draft: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Draft i is kept, after all before it, if ``u[i] * q(token) < p(token)``; one token
    more is drawn with ``r[b]``, from what the target's row has over the draft's where one
    was not kept, else from the target's last row.

    target: [drafts + batch, vocab] probabilities (float32 or bfloat16, any row stride);
    drafted: int32 [drafts]; start: int32 [batch + 1]; u: float32 [drafts] and r: float32 [batch]
    in [0, 1); draft: [drafts, vocab] of the target's type, or None for drafts that were taken
    greedily.  At most ``width - 1`` drafts of a sequence are looked at.

    Returns int32 ``tokens`` [batch, width], the kept drafts and the drawn token, -1 behind,
    and ``count`` [batch], how many there are."""
    if not target.is_cuda or target.dtype not in _TYPES or target.dim() != 2:
        raise ValueError("target must be [rows, vocab] float32 or bfloat16 on a CUDA device")
    device, vocab = target.device, target.shape[1]
    if _current_device() != device.index:
        with torch.cuda.device(device.index):
            return verify(target, drafted, start, u, r, width=width, draft=draft)
    if drafted.dim() != 1 or r.dim() != 1:
        raise ValueError("drafted and r must have one dimension")
    n, batch, i32, f32 = drafted.shape[0], r.shape[0], torch.int32, torch.float32
    if drafted.dtype is not i32 or start.dtype is not i32 or u.dtype is not f32 or r.dtype is not f32 or \
            start.shape != (batch + 1,) or u.shape != (n,) or drafted.device != device or start.device != device or \
            u.device != device or r.device != device or not (drafted.is_contiguous() and start.is_contiguous() and
                                                             u.is_contiguous() and r.is_contiguous()):
        raise ValueError(f"drafted [{n}] and start [{batch + 1}] must be contiguous int32, u [{n}] and r [{batch}] "
                         f"contiguous float32, all on {device}")
    if not 1 <= width <= 1 << 20:
        raise ValueError("width must lie between 1 and 2^20")
    ld = _rows(target, n + batch, vocab, target.dtype, device, "target")
    ld_draft = 0 if draft is None else _rows(draft, n, vocab, target.dtype, device, "draft")
    tokens = torch.empty((batch, width), dtype=torch.int32, device=device)
    count = torch.empty((batch,), dtype=torch.int32, device=device)
    capi.pipo_op_verify_drafts(_TYPES[target.dtype], vocab, batch, n, target.data_ptr(), ld,
                               0 if draft is None else draft.data_ptr(), ld_draft, drafted.data_ptr(), start.data_ptr(),
                               u.data_ptr(), r.data_ptr(), width, tokens.data_ptr(), count.data_ptr(),
                               _raw_stream(device.index))
    return tokens, count
