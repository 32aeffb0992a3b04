"""8-bit paged batches for the tests, and the definitions of the operators around them,
written without the library: codes and scales in 64 bits, block tables request by request,
verification token by token in whole numbers."""
import copy
import math

import torch

from paged_util import PAGE, Batch

TOP = 448.0


def scale_of(most: float) -> float:
    """The power of two that leaves `most` in [32, 64), within [2^-100, 2^7]."""
    return 2.0 ** min(max(math.frexp(most)[1] - 6, -100), 7) if most > 0 else 2.0 ** -100


def codes_of(x):
    """x (fp64, already divided by the scale) as e4m3 codes, rounded once: the 64-bit values go through
    fp32 exactly where the tests need equal codes."""
    return x.clamp(-TOP, TOP).float().to(torch.float8_e4m3fn)


class Batch8:
    """A Batch whose pools are codes (k8, v8) with scales; `plain` is the same batch with
    the values that they stand for, in fp64."""

    def __init__(self, lens, new, n_q, n_kv, d_h, seed=0, k_mult=None, v_mult=None, **kw):
        x = Batch(lens, new, n_q, n_kv, d_h, torch.float32, seed=seed, **kw)
        self.x, self.q = x, x.q.bfloat16()
        self.table, self.q_start, self.kv_len, self.tokens = x.table, x.q_start, x.kv_len, x.tokens
        g = torch.Generator().manual_seed(seed + 1)
        pools = []
        for pool, mult in ((x.k, k_mult), (x.v, v_mult)):
            y = pool.double()
            if mult is not None:  # exponents of the blocks' magnitudes
                y = y * 2.0 ** torch.randint(mult[0], mult[1] + 1, (x.blocks, n_kv, 1, 1), generator=g).double()
            most = y.nan_to_num(0.0).abs().amax((2, 3))
            s = torch.tensor([[scale_of(m) for m in row] for row in most.tolist()])
            pools.append((codes_of(y / s[..., None, None].double()), s))
        (self.k8, self.k_scale), (self.v8, self.v_scale) = pools
        self.plain = copy.copy(x)
        self.plain.q = self.q
        self.plain.k = self.k8.double() * self.k_scale[..., None, None].double()
        self.plain.v = self.v8.double() * self.v_scale[..., None, None].double()


def put(codes, scale, table_row, old_len, x):
    """Append x [entries, heads, d] (fp64) behind old_len entries of a sequence, block by block; codes as fp64
    values (code * 1), changed in place like the scales (fp64)."""
    n = x.shape[0]
    for p in range(old_len // PAGE, (old_len + n - 1) // PAGE + 1):
        blk, lo = int(table_row[p]), max(0, old_len - p * PAGE)
        part = x[max(0, p * PAGE - old_len):(p + 1) * PAGE - old_len]
        for g in range(x.shape[1]):
            y = part[:, g]
            most = float(y.abs().masked_fill(~y.isfinite(), 0).max())
            if lo == 0 or most > TOP * float(scale[blk, g]):
                s = scale_of(most)
                if lo:
                    codes[blk, g, :lo] = codes_of(codes[blk, g, :lo] * (float(scale[blk, g]) / s)).double()
                scale[blk, g] = s
            codes[blk, g, lo:lo + y.shape[0]] = codes_of(y / float(scale[blk, g])).double()


def tables(table, held, free, n_free, kept, added, tokens):
    """A step's tables, request by request (lists; table, held and free are changed in place)."""
    width = len(table[0])
    asked = []
    stack = free[:n_free]
    for b in range(len(kept)):
        keep = min(max(kept[b], 0), PAGE * held[b])
        first = -(-keep // PAGE)
        for p in range(first, held[b]):
            stack.append(table[b][p])
            table[b][p] = -1
        held[b] = first
        asked.append((keep, max(added[b], 0), first))
    free[:len(stack)] = stack
    blocks = room = 0
    given = []
    for keep, add, first in asked:
        want = -(-(keep + add) // PAGE) - first
        if first + want > width:
            given.append(None)
            continue
        blocks += want
        room += add
        given.append(want if (want == 0 or blocks <= len(stack)) and room <= tokens else None)
    left = len(stack) - sum(w for w in given if w)
    at, q_start, kv_len, slots, positions = left, [0], [], [], []
    for b, ((keep, add, first), want) in enumerate(zip(asked, given)):
        if want is None:
            add = want = 0
        for p in range(first, first + want):
            table[b][p] = stack[at]
            at += 1
        held[b] = first + want
        for pos in range(keep, keep + add):
            slots.append(table[b][pos // PAGE] * PAGE + pos % PAGE)
            positions.append(pos)
        kv_len.append(keep + add)
        q_start.append(q_start[-1] + add)
    pad = [-1] * (tokens - len(slots))
    return left, q_start, kv_len, slots + pad, positions + pad


def weight(x: float) -> int:
    """A probability as a multiple of 2^-44, ties to even."""
    return 0 if math.isnan(x) or x <= 0 else round(min(x, 1.0) * 2 ** 44)


def verify(target, drafted, start, u, r, width, draft=None):
    """Kept drafts and the drawn token of every sequence: Python numbers, no sums of floating-point values."""
    f32 = lambda x: x.float()  # noqa: E731
    vocab, out, counts = target.shape[1], [], []
    start, drafted = start.tolist(), drafted.tolist()
    for b in range(len(start) - 1):
        row, rest, n = [], None, min(start[b + 1] - start[b], width - 1)
        for i in range(n):
            p, t = f32(target[start[b] + b + i]), drafted[start[b] + i]
            ok = 0 <= t < vocab
            if ok:
                q = 1.0 if draft is None else float(draft[start[b] + i, t])
                ok = float(u[start[b] + i]) * q < float(p[t])  # (24 bits times 24 bits: exact in 64)
            if not ok:
                if draft is not None:
                    rest = p - f32(draft[start[b] + i])
                else:
                    rest = p.clone()
                    if 0 <= t < vocab:
                        rest[t] = 0
                break
            row.append(t)
        p = f32(target[start[b] + b + len(row)])
        w = [weight(x) for x in (p if rest is None else rest).tolist()]
        if sum(w) == 0:
            w = [weight(x) for x in p.tolist()]
        goal = int(float(r[b]) * float(sum(w)))
        total = 0
        for v, x in enumerate(w):
            total += x
            if total > goal:
                break
        counts.append(len(row) + 1)
        row.append(v)
        out.append(row + [-1] * (width - len(row)))
    return torch.tensor(out, dtype=torch.int32), torch.tensor(counts, dtype=torch.int32)
