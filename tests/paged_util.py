"""Ragged paged batches for the paged-cache tests, and the operators' definitions
in 64 bits, token by token, written without the library."""
import math

import numpy as np
import torch

PAGE = 64


class Batch:
    """Sequences of lens[b] entries, the last new[b] of them new, in shuffled
    blocks of a pool.  Slots no sequence holds are `junk` (NaN by default), and
    so are the table entries past a sequence's pages."""

    def __init__(self, lens, new, n_q, n_kv, d_h, dtype, seed=0, width=None, junk=float("nan"), spare=2):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new, self.n_q, self.n_kv, self.d_h, self.dtype = list(lens), list(new), n_q, n_kv, d_h, dtype
        nb = len(self.lens)
        pages = [-(-n // PAGE) for n in self.lens]
        self.width = width or max(1, max(pages))
        self.blocks = sum(pages) + spare
        order = torch.randperm(self.blocks, generator=g).tolist()
        table = torch.full((nb, self.width), 1 << 30, dtype=torch.int32)
        self.k = torch.full((self.blocks, n_kv, PAGE, d_h), junk, dtype=dtype)
        self.v = torch.full((self.blocks, n_kv, PAGE, d_h), junk, dtype=dtype)
        at = 0
        for b, n in enumerate(self.lens):
            for p in range(pages[b]):
                blk = order[at]
                at += 1
                table[b, p] = blk
                m = min(PAGE, n - p * PAGE)
                self.k[blk, :, :m] = torch.randn(n_kv, m, d_h, generator=g).to(dtype)
                self.v[blk, :, :m] = torch.randn(n_kv, m, d_h, generator=g).to(dtype)
        self.table = table
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum(self.new)]), dtype=torch.int32)
        self.kv_len = torch.tensor(self.lens, dtype=torch.int32)
        self.tokens = int(sum(self.new))
        self.q = (2.0 * torch.randn(self.tokens, n_q, d_h, generator=g)).to(dtype)
        self.g = g

    def each_token(self):
        """(row, sequence, position); the position is negative without an entry."""
        t = 0
        for b, n in enumerate(self.new):
            for i in range(n):
                yield t, b, self.lens[b] - n + i
                t += 1

    def rows(self, pool, b, g, idx):
        """Entries idx (an int64 tensor) of sequence b, head g, in fp64."""
        blk = self.table[b].long()[idx // PAGE]
        return pool[blk, g, idx % PAGE].double()


def ref_attend(x: Batch, scale, window=0, pages=None):
    out = torch.zeros(x.tokens, x.n_q, x.d_h, dtype=torch.float64)
    grp = x.n_q // x.n_kv
    for t, b, pos in x.each_token():
        if pos < 0:
            continue
        for g in range(x.n_kv):
            j = torch.arange(max(0, pos - window + 1) if window else 0, pos + 1)
            if pages is not None:
                keep = set(pages[t, g].tolist())
                j = j[torch.isin(j // PAGE, torch.tensor(sorted(keep)))]
            if len(j) == 0:
                continue
            kk, vv = x.rows(x.k, b, g, j), x.rows(x.v, b, g, j)
            q = x.q[t, g * grp:(g + 1) * grp].double()
            out[t, g * grp:(g + 1) * grp] = torch.softmax(scale * q @ kk.T, -1) @ vv
    return out


def ref_scores(x: Batch, means, scale):
    out = torch.full((x.tokens, x.n_kv, x.width), -math.inf, dtype=torch.float64)
    grp = x.n_q // x.n_kv
    for t, b, pos in x.each_token():
        for p in range(pos // PAGE + 1 if pos >= 0 else 0):
            for g in range(x.n_kv):
                q = x.q[t, g * grp:(g + 1) * grp].double().sum(0)
                out[t, g, p] = scale * (q * means[x.table[b, p].item(), g].double()).sum()
    return out


def ref_select(x: Batch, scores, top, sink, local):
    """The kept pages by sorting: forced ones, then by (score, lower page)."""
    out = torch.full((x.tokens, x.n_kv, top), -1, dtype=torch.int32)
    for t, b, pos in x.each_token():
        seen = pos // PAGE + 1 if pos >= 0 else 0
        for g in range(x.n_kv):
            sc = [float(s) for s in scores[t, g, :seen]]
            fixed = [p for p in range(seen) if p < sink or p >= seen - local]
            rest = [p for p in range(seen) if p not in fixed]
            rest.sort(key=lambda p: (math.isnan(sc[p]), -sc[p] if not math.isnan(sc[p]) else 0.0, p))
            keep = sorted(fixed + rest[:max(0, top - len(fixed))])[:top]
            out[t, g, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
    return out


def ref_append(x: Batch, q, k, v, q_gain, k_gain, eps, theta):
    """(queries, keys, values) of the new tokens in 64 bits; theta None: no rotation."""
    def unit(y, gain):
        y = y.double()
        return y if gain is None else y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gain.double()

    pos = torch.tensor([p for _, _, p in x.each_token()], dtype=torch.float64)

    def turn(y):
        if theta is None:
            return y
        half = x.d_h // 2
        a = pos[:, None] * theta ** (-2.0 * torch.arange(half, dtype=torch.float64) / x.d_h)
        z = torch.complex(y[..., :half], y[..., half:]) * torch.polar(torch.ones_like(a), a)[:, None]
        return torch.cat([z.real, z.imag], -1)

    return turn(unit(q, q_gain)), turn(unit(k, k_gain)), v.double()
