"""The paged-cache operators of ``include/pipo.h`` on torch tensors.

``PagedCache`` describes pools and a block table that the caller owns and
makes the four calls of an attention layer on its device's current CUDA stream:

    cache = PagedCache(k_pool, v_pool, table, n_q=32, means=means)
    q = cache.append(q, k, v, q_start, kv_len, q_gain=..., k_gain=..., rope=...)
    out = cache.attend(q, q_start, kv_len)
    scores = cache.page_scores(q, q_start, kv_len)
    out, pages = cache.attend_pages(q, scores, q_start, kv_len, top=32, sink=1, local=2)

The new tokens of sequence b are rows ``q_start[b] .. q_start[b+1]-1`` of the
token tensors ``[tokens, heads, d_h]`` (any token stride; the heads of a token
back to back), and ``kv_len[b]`` counts its cached entries, the new ones
included.  ``q_start`` and ``kv_len`` are int32 tensors on the device and are
read there: the calls neither synchronise nor depend on host copies, and a
captured graph follows their values.  There is no backward pass: inputs that
require gradients are refused unless gradients are off (``torch.no_grad``).
Shapes and types are checked here, everything else by the library
(``capi.PipoError``).
"""
from __future__ import annotations

import threading
from typing import Dict, Optional, Tuple

import torch

from . import capi

PAGE = 64
_raw_stream = torch._C._cuda_getCurrentRawStream  # the current stream's handle, without a Stream object
_current_device = torch._C._cuda_getDevice
_TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _int32(n: int) -> int:
    """The nearest integer that the library's int32 arguments hold (ctypes would drop the upper bits)."""
    return n if -0x80000000 <= n <= 0x7fffffff else 0x7fffffff if n > 0 else -0x80000000


def rope_table(n: int, d_h: int, theta: float, device="cuda") -> torch.Tensor:
    """(cos, sin) of every position and pair, angle ``position * theta^(-2i/d_h)``,
    computed in fp64 and rounded once: fp32 [n, d_h/2, 2]."""
    i = torch.arange(0, d_h, 2, device=device, dtype=torch.float64)
    a = torch.arange(n, device=device, dtype=torch.float64)[:, None] * theta ** (-i / d_h)
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _no_backward(name: str, x: torch.Tensor) -> None:
    if x.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, and the paged-cache operators have none")


class PagedCache:
    """Pools ``k``, ``v`` [n_blocks, n_kv, 64, d_h] (bf16 or fp32), the block
    table [batch, max_pages] (int32) and, for the page scores, the mean keys
    ``means`` [n_blocks, n_kv, d_h] that ``append`` maintains.  The tensors stay
    the caller's; nothing is copied.  ``attend`` and ``attend_pages`` keep a
    scratch buffer per stream; a call that ``torch.cuda.graph`` captures takes
    one from the graph's own pool instead, which lasts as long as the graph, so that
    later calls, whatever their size, leave its replays alone.  Threads may
    share an object."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, n_q: int,
                 means: Optional[torch.Tensor] = None):
        if k.dtype not in _TYPES or v.dtype != k.dtype or k.dim() != 4 or k.shape != v.shape or k.shape[2] != PAGE \
                or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError("pools must be contiguous [n_blocks, n_kv, 64, d_h] of one type (float32 or bfloat16)")
        if table.dtype != torch.int32 or table.dim() != 2 or not table.is_contiguous():
            raise ValueError("the block table must be a contiguous int32 [batch, max_pages]")
        if means is not None and (means.dtype != k.dtype or not means.is_contiguous() or
                                  means.shape != (k.shape[0], k.shape[1], k.shape[3])):
            raise ValueError("means must be contiguous [n_blocks, n_kv, d_h] of the pools' type")
        if not k.is_cuda or any(t.device != k.device for t in (v, table) + (() if means is None else (means,))):
            raise ValueError("pools, table and means must be on one CUDA device")
        self.k, self.v, self.table, self.means = k, v, table, means
        self.n_q, self.n_kv, self.d_h, self.dtype, self.device = n_q, k.shape[1], k.shape[3], k.dtype, k.device
        self.index = k.device.index
        self._c = capi.pipo_paged(_TYPES[k.dtype], _int32(n_q), k.shape[1], k.shape[3], PAGE, k.shape[0],
                                  table.shape[1], table.shape[0], k.data_ptr(), v.data_ptr(),
                                  None if means is None else means.data_ptr(), table.data_ptr())
        self._seqs = table.shape[0]
        self._lock = threading.Lock()
        self._buffers: Dict[int, torch.Tensor] = {}  # scratch by stream
        self._need, self._need_for = 0, -1           # scratch bytes of the last token count

    # ---- arguments

    def _batch(self, q_start: torch.Tensor, kv_len: torch.Tensor) -> None:
        n, i32 = self._seqs, torch.int32
        if q_start.dtype is not i32 or kv_len.dtype is not i32 or q_start.shape != (n + 1,) or kv_len.shape != (n,) or \
                not (q_start.is_contiguous() and kv_len.is_contiguous()) or q_start.device != self.device or \
                kv_len.device != self.device:
            raise ValueError(f"q_start [{n + 1}] and kv_len [{n}] must be contiguous int32 on the pools' device")
        self._c.q_start, self._c.kv_len = q_start.data_ptr(), kv_len.data_ptr()

    def _rows(self, x: torch.Tensor, heads: int, name: str, dtype: torch.dtype) -> int:
        """Token stride of [tokens, heads, d_h] with the heads back to back."""
        shape, stride = x.shape, x.stride()
        if len(shape) != 3 or shape[1] != heads or shape[2] != self.d_h or x.dtype is not dtype or \
                x.device != self.device or (shape[0] and (stride[2] != 1 or (heads > 1 and stride[1] != self.d_h))):
            raise ValueError(f"{name} must be [tokens, {heads}, {self.d_h}] {dtype} with whole rows")
        _no_backward(name, x)
        return stride[0] if shape[0] > 1 else heads * self.d_h

    def _work(self, tokens: int, stream: int) -> torch.Tensor:
        """Scratch of a call on the current stream (``stream``).  A buffer is allocated on
        the stream that uses it: an outgrown one goes back behind that stream's work.  Under a
        capture it is new: the graph's pool keeps it for the replays, and calls of
        one capture take the same memory in turn."""
        if self._need_for != tokens:
            self._need = max(capi.pipo_op_attn_paged_scratch(self._c, tokens), 16)
            self._need_for = tokens
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(self._need, dtype=torch.uint8, device=self.device)
        buf = self._buffers.get(stream)
        if buf is None or buf.numel() < self._need:
            buf = self._buffers[stream] = torch.empty(self._need, dtype=torch.uint8, device=self.device)
        return buf

    @property
    def _scratch(self) -> Optional[torch.Tensor]:
        """The current stream's buffer, if it has one."""
        return self._buffers.get(_raw_stream(self.index))

    # ---- the calls.  The library plans and launches on the thread's current device, so that each
    # makes that the pools' first; and it reads the object's description of the batch without
    # the interpreter lock, so that the calls of an object take turns from there on.

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, q_start: torch.Tensor,
               kv_len: torch.Tensor, *, q_gain: Optional[torch.Tensor] = None,
               k_gain: Optional[torch.Tensor] = None, eps: float = 1e-6, rope: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Normalise (where a gain is given) and rotate (where a table is) the
        new queries and keys, append keys and values, update the page means.
        Returns the queries [tokens, n_q, d_h] in the pools' type (None without q)."""
        if _current_device() != self.index:
            with torch.cuda.device(self.index):
                return self.append(q, k, v, q_start, kv_len, q_gain=q_gain, k_gain=k_gain, eps=eps, rope=rope, out=out)
        if k.dtype not in _TYPES:
            raise ValueError("keys must be float32 or bfloat16")
        tokens = k.shape[0]
        ld_k, ld_v = self._rows(k, self.n_kv, "k", k.dtype), self._rows(v, self.n_kv, "v", k.dtype)
        ld_q = self._rows(q, self.n_q, "q", k.dtype) if q is not None else 0
        if v.shape[0] != tokens or (q is not None and q.shape[0] != tokens):
            raise ValueError("q, k and v must have the same number of tokens")
        for gain in (q_gain, k_gain):
            if gain is None:
                continue
            if gain.dtype != self.dtype or gain.shape != (self.d_h,) or not gain.is_contiguous() or \
                    gain.device != self.device:
                raise ValueError("gains must be [d_h] of the pools' type")
            _no_backward("a gain", gain)
        if rope is not None:
            if rope.dtype != torch.float32 or rope.dim() != 3 or rope.shape[1] != self.d_h // 2 or \
                    rope.shape[2] != 2 or not rope.is_contiguous() or rope.device != self.device:
                raise ValueError("rope must be a contiguous float32 [positions, d_h / 2, 2]")
            _no_backward("rope", rope)
        if q is None:
            out = None
        elif out is None:
            out = torch.empty((tokens, self.n_q, self.d_h), dtype=self.dtype, device=self.device)
        elif out.shape != (tokens, self.n_q, self.d_h) or out.dtype != self.dtype or not out.is_contiguous() or \
                out.device != self.device:
            raise ValueError("out must be a contiguous [tokens, n_q, d_h] of the pools' type")
        p = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
        with self._lock:
            self._batch(q_start, kv_len)
            capi.pipo_op_kv_append(self._c, tokens, _TYPES[k.dtype], p(q), ld_q, k.data_ptr(), ld_k, v.data_ptr(),
                                   ld_v, p(q_gain), p(k_gain), eps, p(rope), 0 if rope is None else rope.shape[0],
                                   p(out), _raw_stream(self.index))
        return out

    def _out(self, q: torch.Tensor, out: Optional[torch.Tensor]) -> Tuple[torch.Tensor, int]:
        if out is None:
            out = torch.empty((q.shape[0], self.n_q, self.d_h), dtype=self.dtype, device=self.device)
            return out, self.n_q * self.d_h
        if out.shape[0] != q.shape[0]:
            raise ValueError("out must have a row for every token")
        return out, self._rows(out, self.n_q, "out", self.dtype)

    def attend(self, q: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, *,
               scale: Optional[float] = None, window: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Causal attention of the new tokens over the cache; ``window`` > 0
        keeps the last ``window`` entries of every token, and pages that it has
        passed for all new tokens of a sequence are not needed (their blocks
        and table entries may hold anything).  scale: 1/sqrt(d_h) unless given."""
        if _current_device() != self.index:
            with torch.cuda.device(self.index):
                return self.attend(q, q_start, kv_len, scale=scale, window=window, out=out)
        ld_q = self._rows(q, self.n_q, "q", self.dtype)
        out, ld_out = self._out(q, out)
        stream = _raw_stream(self.index)
        with self._lock:
            self._batch(q_start, kv_len)
            w = self._work(q.shape[0], stream)
            capi.pipo_op_attn_paged(self._c, q.shape[0], q.data_ptr(), ld_q,
                                    self.d_h ** -0.5 if scale is None else scale, _int32(window), out.data_ptr(),
                                    ld_out, w.data_ptr(), w.numel(), stream)
        return out

    def page_scores(self, q: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, *,
                    scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """fp32 [tokens, n_kv, max_pages]: the score of every page a token sees,
        -inf for the others."""
        if self.means is None:
            raise ValueError("page scores need a cache with means")
        if _current_device() != self.index:
            with torch.cuda.device(self.index):
                return self.page_scores(q, q_start, kv_len, scale=scale, out=out)
        ld_q = self._rows(q, self.n_q, "q", self.dtype)
        shape = (q.shape[0], self.n_kv, self.table.shape[1])
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=self.device)
        elif out.shape != shape or out.dtype != torch.float32 or not out.is_contiguous() or out.device != self.device:
            raise ValueError("out must be a contiguous float32 [tokens, n_kv, max_pages]")
        with self._lock:
            self._batch(q_start, kv_len)
            capi.pipo_op_page_scores(self._c, q.shape[0], q.data_ptr(), ld_q,
                                     self.d_h ** -0.5 if scale is None else scale, out.data_ptr(),
                                     _raw_stream(self.index))
        return out

    def attend_pages(self, q: torch.Tensor, scores: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor, *,
                     top: int, sink: int = 1, local: int = 1, scale: Optional[float] = None,
                     out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Causal attention over ``top`` pages per token and kv head: the first
        ``sink``, the last ``local`` and the best scored.  ``local`` >= 1 keeps the
        page a token stands in, whose mean counts later tokens of the same call.  Returns
        the outputs and the pages, int32 [tokens, n_kv, top], ascending, -1 behind the last."""
        if _current_device() != self.index:
            with torch.cuda.device(self.index):
                return self.attend_pages(q, scores, q_start, kv_len, top=top, sink=sink, local=local, scale=scale,
                                         out=out)
        ld_q = self._rows(q, self.n_q, "q", self.dtype)
        if scores.shape != (q.shape[0], self.n_kv, self.table.shape[1]) or scores.dtype != torch.float32 or \
                not scores.is_contiguous() or scores.device != self.device:
            raise ValueError("scores must be a contiguous float32 [tokens, n_kv, max_pages]")
        _no_backward("scores", scores)
        out, ld_out = self._out(q, out)
        pages = torch.empty((q.shape[0], self.n_kv, top), dtype=torch.int32, device=self.device)
        stream = _raw_stream(self.index)
        with self._lock:
            self._batch(q_start, kv_len)
            w = self._work(q.shape[0], stream)
            capi.pipo_op_attn_pages(self._c, q.shape[0], q.data_ptr(), ld_q,
                                    self.d_h ** -0.5 if scale is None else scale, scores.data_ptr(), _int32(top),
                                    _int32(sink), _int32(local), out.data_ptr(), ld_out, pages.data_ptr(),
                                    w.data_ptr(), w.numel(), stream)
        return out, pages
