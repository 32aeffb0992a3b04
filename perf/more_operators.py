"""What the operators of a drafting server with an 8-bit cache are measured on.

Four operators, in the order in which a serving step uses them:

* ``tables``   block tables, lengths and slot maps of a step from the requests'
               lengths: entries that are no longer kept give their blocks back,
               new tokens get blocks, every new token learns its slot;
* ``append8``  per-head RMSNorm of queries and keys, rotate-half rotation, append
               of keys and values to a cache of e4m3 codes with a power of two as
               scale for every block and kv head;
* ``attend8``  causal attention of ragged chunks of new tokens over that cache,
               optionally windowed;
* ``verify``   drafted tokens against the target's probabilities: each is kept
               with probability min(1, p/q) by a given random number, and the
               token behind the last kept one is drawn from max(p - q, 0), or from
               the target's next row when all were kept, by another one.

Head shapes are the repository's models' (4b/9b: 32 query and 8 kv heads of 128)
and generic ones, the vocabulary is theirs (151936; tiny: 4096) or generic.
Keys and queries are as a per-head norm leaves them, values N(0, 1).
"""
import math

import numpy as np
import torch

own = False

PAGE = 64
TOP = 448.0            # largest e4m3 value
LOW, HIGH = -100, 7    # exponents that a block's scale may have
UNIT = 2.0 ** 44       # probabilities are added up as whole multiples of 1 / UNIT
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _cache(name, op, n_q, n_kv, d_h, batch, ctx, new, ragged, **kw):
    return dict(name=name, op=op, n_q=n_q, n_kv=n_kv, d_h=d_h, batch=batch, ctx=ctx, new=new, ragged=ragged, **kw)


def _tables(name, batch, ctx, new, short):
    return dict(name=name, op="tables", batch=batch, ctx=ctx, new=new, short=short)


def _verify(name, batch, vocab, drafts, ragged, dtype, greedy):
    return dict(name=name, op="verify", batch=batch, vocab=vocab, drafts=drafts, ragged=ragged, dtype=dtype,
                greedy=greedy)


def listed():
    return [
        # a small server between two steps: decoding users, a few new prompts (latency)
        _tables("tables-b16", 16, 2415, 300, False),
        # a large one that runs out of blocks
        _tables("tables-b1024-short", 1024, 4096, 1024, True),
        # one user decoding (latency)
        _cache("append8-4b-b1", "append8", 32, 8, 128, 1, 1155, 1, False, in_f32=True, norm=True),
        # decoding users and prompts that join, fp32 projections
        _cache("append8-4b-b16-mixed", "append8", 32, 8, 128, 16, 1288, 300, True, in_f32=True, norm=True),
        # two long prompts at once, bf16 activations
        _cache("append8-4b-prompts", "append8", 32, 8, 128, 2, 0, 8191, False, in_f32=False, norm=True),
        # one user (latency)
        _cache("attend8-4b-b1", "attend8", 32, 8, 128, 1, 1155, 1, False, window=0),
        # users with long documents in their caches: the cache's bytes are the time
        _cache("attend8-4b-b8-long", "attend8", 32, 8, 128, 8, 15491, 1, False, window=0),
        # many users, four drafted tokens and the one before each, a sliding window
        _cache("attend8-64-b64-drafts", "attend8", 16, 16, 64, 64, 2415, 5, False, window=1024),
        # the last chunk of a long prompt: the tensor cores' rate is the time
        _cache("attend8-4b-chunk", "attend8", 32, 8, 128, 1, 14336, 2048, False, window=0),
        # one user, the pair's drafted token (latency)
        _verify("verify-4b-b1", 1, 151936, 1, False, "f32", False),
        # many users, up to four drafted tokens each
        _verify("verify-4b-b64", 64, 151936, 4, True, "f32", False),
        # drafts that were taken greedily: no draft probabilities
        _verify("verify-4b-b16-greedy", 16, 151936, 4, False, "f32", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 280)


def _plain_elements(case):
    """Elements of the largest array of the plain form."""
    if case["op"] == "attend8":
        past, new = _lengths(case)
        return case["batch"] * case["n_q"] * max(new) * max(p + n for p, n in zip(past, new))
    if case["op"] == "verify":
        return 4 * case["batch"] * (case["drafts"] + 1) * case["vocab"]
    return 0


def draw(rng):
    op = rng.choice(["tables", "append8", "append8", "attend8", "attend8", "attend8", "verify"])
    if op == "tables":
        c = _tables("", _log(rng, 1, 1024), _log(rng, 16, 16384), _log(rng, 1, 2048), rng.random() < 0.4)
    elif op == "verify":
        vocab = rng.choice([4096, 151936, 151936, _log(rng, 257, 200000)])
        c = _verify("", _log(rng, 1, 256), vocab, rng.randint(1, 12), rng.random() < 0.5,
                    "bf16" if rng.random() < 0.3 else "f32", rng.random() < 0.3)
    else:
        n_q, n_kv, d_h = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 16, 64), (24, 2, 64), (8, 1, 128),
                                     (4, 2, 64)])
        new = 1 if rng.random() < 0.4 else rng.randint(2, 8) if rng.random() < 0.4 else _log(rng, 9, 2048)
        kw = dict(in_f32=rng.random() < 0.5, norm=rng.random() < 0.75) if op == "append8" else \
            dict(window=0 if rng.random() < 0.7 else _log(rng, 16, 4096))
        c = _cache("", op, n_q, n_kv, d_h, _log(rng, 1, 64), _log(rng, 16, 16384), new, rng.random() < 0.5, **kw)
    del c["name"]
    most = max(_cost(x) for x in listed() if x["op"] == op)
    while _cost(c) > most or _plain_elements(c) > 1_100_000_000:
        if c["batch"] > 1:
            c["batch"] = c["batch"] * 2 // 3
        elif c.get("new", 1) > 1:
            c["new"] = c["new"] * 2 // 3
        elif op == "verify":
            c["drafts"] = c["drafts"] * 2 // 3
        else:
            c["ctx"] = c["ctx"] * 2 // 3
    return c


def _lengths(case):
    """(cached entries, new tokens) of every sequence.  Ragged: ages spread up
    to ctx, every other sequence decodes one token, the others bring chunks of
    different lengths, and one of four and more is idle (no new token)."""
    n, ctx, new = case["batch"], case["ctx"], case["new"]
    if not case["ragged"]:
        return [ctx] * n, [new] * n
    past = [ctx * ((b * 7 + 3) % n + 1) // n for b in range(n)]
    count = [1 if b % 2 else 1 + (new - 1) * ((b * 5 + 1) % n + 1) // n for b in range(n)]
    if n >= 4:
        count[n // 2] = 0
    return past, count


def _requests(case):
    """Entries held, entries kept and new tokens of every request: most decode one to
    five tokens after up to four rejected ones, every eighth has ended and its place takes a
    new prompt, every seventh pauses."""
    n, ctx, new = case["batch"], case["ctx"], case["new"]
    held = [1 + ctx * ((b * 7 + 3) % n + 1) // n for b in range(n)]
    kept = [0 if b % 8 == 5 else max(0, h - b % 5) for b, h in enumerate(held)]
    added = [1 + new * ((b * 5 + 1) % n) // n if b % 8 == 5 else 0 if b % 7 == 6 else 1 + b * 3 % 5 for b in range(n)]
    return held, kept, added


def _counts(case):
    """Drafted tokens of every sequence."""
    n, d = case["batch"], case["drafts"]
    return [(b * 5 + 1) % (d + 1) for b in range(n)] if case["ragged"] else [d] * n


def _visible(case):
    """Per new token: the entries it may attend to, as (first, last + 1)."""
    w = case["window"]
    for p, n in zip(*_lengths(case)):
        for i in range(n):
            yield max(0, p + i + 1 - w) if w else 0, p + i + 1


def _pages(n):
    return -(-n // PAGE)


def work(case):
    op = case["op"]
    if op == "tables":
        held, kept, added = _requests(case)
        moved = sum(abs(_pages(h) - _pages(k)) + _pages(k + a) - _pages(k) for h, k, a in zip(held, kept, added))
        # lengths in and out, blocks given back and taken (stack and table), two numbers a token
        return {"bytes": 4 * (5 * case["batch"] + 2 * moved + 2 * sum(added)), "flops": 0}
    if op == "verify":
        # the target's row that the last token is drawn from (a draft row besides, where one was
        # rejected: not counted), and a few numbers per drafted token
        es = 4 if case["dtype"] == "f32" else 2
        by = case["batch"] * (case["vocab"] * es + 4 * (case["drafts"] + 2))
        return {"bytes": by + sum(_counts(case)) * (8 + 2 * es), "flops": 2 * case["batch"] * case["vocab"]}
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d_h"]
    past, new = _lengths(case)
    t = sum(new)
    if op == "append8":
        by = t * (n_q + 2 * n_kv) * d * (4 if case["in_f32"] else 2) + t * n_q * d * 2 + t * 2 * n_kv * d + t * d * 4
        by += 8 * sum((p + n - 1) // PAGE - p // PAGE + 1 for p, n in zip(past, new) if n) * n_kv
        return {"bytes": by, "flops": t * (n_q + n_kv) * d * 8}
    w = case["window"]
    seen = [p + n - (max(0, p + 1 - w) if w else 0) for p, n in zip(past, new) if n]
    pairs = sum(b - a for a, b in _visible(case))
    return {"bytes": 4 * t * n_q * d + 2 * sum(seen) * n_kv * d + 8 * n_kv * sum(_pages(x) for x in seen),
            "flops": 4 * d * n_q * pairs}


def _encode(x):
    """x [blocks, heads, PAGE, d] as e4m3 codes with a scale for every block and head."""
    scale = _scale_of(x.abs().amax((2, 3)))
    return (x / scale[..., None, None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn), scale


def _scale_of(most):
    """The power of two that leaves the largest magnitude in [32, 64); the smallest one for zeros."""
    e = torch.frexp(most)[1] - 6
    e = torch.where(most > 0, e, torch.full_like(e, LOW)).clamp(LOW, HIGH)
    return torch.ldexp(torch.ones_like(most), e)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    randn = lambda *shape: torch.randn(*shape, generator=g, device=dev)  # noqa: E731
    if case["op"] == "tables":
        held, kept, added = _requests(case)
        width = max(_pages(max(h, k + a)) for h, k, a in zip(held, kept, added))
        pages = [_pages(h) for h in held]
        need = sum(_pages(k + a) - _pages(k) for k, a in zip(kept, added))
        back = sum(p - _pages(k) for p, k in zip(pages, kept))
        spare = max(0, (need - back) * 2 // 3) if case["short"] else need + 7
        blocks = sum(pages) + spare
        order = torch.randperm(blocks, generator=g, device=dev).to(torch.int32)
        held_pages = ints(pages)
        at = torch.cumsum(held_pages, 0)[:, None] - held_pages[:, None] + torch.arange(width, device=dev)
        table = torch.where(torch.arange(width, device=dev) < held_pages[:, None], order[at.clamp(max=blocks - 1)], -1)
        free = torch.full((blocks,), -1, dtype=torch.int32, device=dev)
        free[:spare] = order[sum(pages):]
        return dict(case=case, table=table.to(torch.int32).contiguous(), held=held_pages, free=free,
                    n_free=ints([spare]), kept=ints(kept), added=ints(added), tokens=sum(added) + 3)
    if case["op"] == "verify":
        count, vocab, dt = _counts(case), case["vocab"], TYPES[case["dtype"]]
        t, n = sum(count), case["batch"]
        logits = randn(t + n, vocab) * 2.5
        first = np.cumsum([0] + count)
        rows = torch.tensor([first[b] + b + i for b in range(n) for i in range(count[b])], dtype=torch.long, device=dev)
        drafts = torch.softmax(logits[rows] + 0.8 * randn(t, vocab), -1)
        drafted = torch.argmax(drafts, -1) if case["greedy"] or not t else \
            torch.multinomial(drafts, 1, generator=g)[:, 0]
        rand = lambda k: torch.rand(k, generator=g, device=dev)  # noqa: E731
        return dict(case=case, target=torch.softmax(logits, -1).to(dt),
                    draft=None if case["greedy"] else drafts.to(dt), drafted=drafted.to(torch.int32),
                    start=ints(first.tolist()), u=rand(t), r=rand(n))
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d_h"]
    past, new = _lengths(case)
    t = sum(new)
    width = _pages(max(p + n for p, n in zip(past, new)))
    blocks = case["batch"] * width + 3
    k, ks = _encode(randn(blocks, n_kv, PAGE, d))
    v, vs = _encode(randn(blocks, n_kv, PAGE, d))
    s = dict(case=case, k=k, v=v, k_scale=ks, v_scale=vs,
             table=torch.randperm(blocks, generator=g, device=dev)[:case["batch"] * width]
             .reshape(case["batch"], width).to(torch.int32),
             q_start=ints([0] + np.cumsum(new).tolist()), kv_len=ints([p + n for p, n in zip(past, new)]),
             most_new=max(new), scale=d ** -0.5)
    if case["op"] == "append8":
        # queries, keys and values as one projection leaves them: a row per token
        s["qkv"] = (randn(t, n_q + 2 * n_kv, d) * 2.0).to(torch.float32 if case["in_f32"] else torch.bfloat16)
        s["q_gain"] = (1 + 0.1 * randn(d)).bfloat16() if case["norm"] else None
        s["k_gain"] = (1 + 0.1 * randn(d)).bfloat16() if case["norm"] else None
        ang = torch.arange(width * PAGE, device=dev, dtype=torch.float64)[:, None] \
            * (1.0e6 ** (-torch.arange(0, d, 2, device=dev, dtype=torch.float64) / d))
        s["rope"] = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()
        s["eps"] = 1e-6
    else:
        s["q"] = (randn(t, n_q, d) * (1.0 + 0.5 * (torch.arange(n_q, device=dev) % 3))[:, None]).bfloat16()
    return s


# ---- the plain forms: elementary torch operations ------------------------------

def _plain_tables(s):
    table, free, tokens = s["table"], s["free"], s["tokens"]
    dev, width, blocks = table.device, table.shape[1], free.shape[0]
    held, add, n_free = s["held"].long(), s["added"].long().clamp(min=0), s["n_free"].long()
    keep = torch.minimum(s["kept"].long().clamp(min=0), PAGE * held)
    kp = (keep + PAGE - 1) // PAGE
    want = (keep + add + PAGE - 1) // PAGE
    fit = want <= width
    want = torch.where(fit, want - kp, 0)
    rel = held - kp
    top = n_free + rel.sum()
    ok = fit & ((want == 0) | (want.cumsum(0) <= top)) & (torch.where(fit, add, 0).cumsum(0) <= tokens)
    take, n = torch.where(ok, want, 0), torch.where(ok, add, 0)
    col = torch.arange(width, device=dev)
    # blocks given back go onto the stack, request by request
    gone = (col >= kp[:, None]) & (col < held[:, None])
    at = n_free + (rel.cumsum(0) - rel)[:, None] + col - kp[:, None]
    stack = torch.cat([free, free.new_zeros(1)])
    stack[torch.where(gone, at, blocks)] = table
    free.copy_(stack[:blocks])
    # the new ones are its last, in the same order
    left = top - take.sum()
    new = (col >= kp[:, None]) & (col < (kp + take)[:, None])
    at = left + (take.cumsum(0) - take)[:, None] + col - kp[:, None]
    table.copy_(torch.where(new, free[torch.where(new, at, 0)], torch.where(gone, -1, table)))
    s["held"].copy_(kp + take)
    s["n_free"].copy_(left)
    q_start = torch.cat([n.new_zeros(1), n.cumsum(0)])
    t = torch.arange(tokens, device=dev)
    b = torch.searchsorted(q_start[1:].contiguous(), t, right=True)
    live = b < n.shape[0]
    b = b.clamp(max=n.shape[0] - 1)
    pos = torch.where(live, keep[b] + t - q_start[b], 0)
    slot = table.long()[b, pos // PAGE] * PAGE + pos % PAGE
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return dict(q_start=i32(q_start), kv_len=i32(keep + n), slots=i32(torch.where(live, slot, -1)),
                positions=i32(torch.where(live, pos, -1)), table=table, held=s["held"], free=free, n_free=s["n_free"])


def _tokens(s, t):
    """Sequence, index within it and position of every token."""
    at = torch.arange(t, device=s["k"].device)
    first = s["q_start"].long()
    b = torch.searchsorted(first[1:].contiguous(), at, right=True)
    i = at - first[b]
    return b, i, s["kv_len"].long()[b] - (first[b + 1] - first[b]) + i


def _put(codes, scale, x, page, pos):
    """New entries x [tokens, heads, d] into blocks ``page`` at positions ``pos``."""
    blocks, heads = scale.shape
    idx = page[:, None].expand(-1, heads)
    most = x.abs().masked_fill(~x.isfinite(), 0).amax(-1)
    most = torch.zeros_like(scale).scatter_reduce_(0, idx, most, "amax")
    first = torch.full((blocks,), PAGE, device=x.device).scatter_reduce_(0, page, pos % PAGE, "amin")[:, None]
    # a block keeps its scale while the new entries fit it; the codes it holds move with a new one
    renew = (first < PAGE) & ((first == 0) | (most > TOP * scale))
    fresh = torch.where(renew, _scale_of(most), scale)
    moved = (codes.float() * (scale / fresh)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    move = (renew & (first > 0))[..., None] & (torch.arange(PAGE, device=x.device) < first)[:, None]
    raw = codes.view(torch.uint8)
    raw.copy_(torch.where(move[..., None], moved, raw))
    scale.copy_(fresh)
    new = (x / scale[page][..., None]).clamp(-TOP, TOP).to(torch.float8_e4m3fn)
    raw[page, :, pos % PAGE] = new.view(torch.uint8)


def _plain_append(s):
    c = s["case"]
    n_q, n_kv, d = c["n_q"], c["n_kv"], c["d_h"]
    x = s["qkv"].float()
    q, kn, vn = x[:, :n_q], x[:, n_q:n_q + n_kv], x[:, n_q + n_kv:]
    b, _, pos = _tokens(s, x.shape[0])
    if c["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + s["eps"]) * s["q_gain"].float()
        kn = kn * torch.rsqrt((kn * kn).mean(-1, keepdim=True) + s["eps"]) * s["k_gain"].float()
    cs, sn = s["rope"][pos][:, None, :, 0], s["rope"][pos][:, None, :, 1]
    turn = lambda y: torch.cat([y[..., :d // 2] * cs - y[..., d // 2:] * sn,  # noqa: E731
                                y[..., d // 2:] * cs + y[..., :d // 2] * sn], -1)
    page = s["table"].long()[b, pos // PAGE]
    _put(s["k"], s["k_scale"], turn(kn), page, pos)
    _put(s["v"], s["v_scale"], vn, page, pos)
    return dict(q=turn(q).bfloat16(), k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _plain_attend(s):
    c, q = s["case"], s["q"]
    n_kv, d, grp = c["n_kv"], c["d_h"], c["n_q"] // c["n_kv"]
    t, nb, most = q.shape[0], c["batch"], s["most_new"]
    b, i, _ = _tokens(s, t)
    first = s["q_start"].long()
    n = first[1:] - first[:-1]
    row = torch.arange(most, device=q.device)
    qp = q[(first[:-1, None] + row).clamp(max=t - 1)].float()  # [b, row, head, d]
    qp = qp.reshape(nb, most, n_kv, grp, d).transpose(1, 2).reshape(nb, n_kv, most * grp, d)

    def rows(pool, scale):
        at = s["table"].long()
        x = pool.view(torch.uint8)[at].view(torch.float8_e4m3fn).float() * scale[at][..., None, None]
        return x.transpose(1, 2).reshape(nb, n_kv, -1, d)

    a = qp @ rows(s["k"], s["k_scale"]).transpose(2, 3) * s["scale"]
    pos = (s["kv_len"].long() - n)[:, None] + row
    j = torch.arange(a.shape[-1], device=q.device)
    see = j <= pos[..., None]
    if c["window"]:
        see &= j > pos[..., None] - c["window"]
    a = a.view(nb, n_kv, most, grp, -1).masked_fill_(~see[:, None, :, None], -math.inf)
    a = a.sub_(a.amax(-1, keepdim=True)).exp_()
    a = a.div_(a.sum(-1, keepdim=True))
    o = a.view(nb, n_kv, most * grp, -1) @ rows(s["v"], s["v_scale"])
    o = o.view(nb, n_kv, most, grp, d).transpose(1, 2)
    return o[b, i].reshape(t, c["n_q"], d).to(q.dtype)


def _plain_verify(s):
    c, dev = s["case"], s["u"].device
    n, vocab, wide = c["batch"], c["vocab"], c["drafts"] + 1
    first = s["start"].long()
    count = first[1:] - first[:-1]
    i = torch.arange(wide, device=dev)
    has = i < count[:, None]
    row = torch.where(has, first[:-1, None] + i, 0)
    if s["drafted"].shape[0]:
        token = torch.where(has, s["drafted"].long()[row], 0)
        p = s["target"][torch.arange(n, device=dev)[:, None] + first[:-1, None] + torch.minimum(i, count[:, None]), token]
        q = torch.ones_like(p) if s["draft"] is None else s["draft"][row, token]
        keep = has & (s["u"][row].double() * q.double() < p.double())
    else:
        token, keep = torch.zeros_like(row), has
    kept = torch.cumprod(keep.long(), 1).sum(1)
    # the row that the last token is drawn from, and what it still holds
    x = s["target"][first[:-1] + torch.arange(n, device=dev) + kept].float()
    res = x
    if s["drafted"].shape[0]:
        at = torch.minimum(first[:-1] + kept, first[-1] - 1)
        if s["draft"] is None:
            hit = torch.arange(vocab, device=dev) == s["drafted"].long()[at][:, None]
            res = torch.where(hit, 0.0, x)
        else:
            res = x - s["draft"][at].float()
        res = torch.where((kept < count)[:, None], res, x)
    # whole numbers, so that the sums do not depend on their order
    whole = lambda y: (y.nan_to_num(0.0).clamp(0, 1).double() * UNIT).round().long().cumsum(1)  # noqa: E731
    cum = whole(res)
    cum = torch.where(cum[:, -1:] > 0, cum, whole(x))
    goal = (s["r"].double() * cum[:, -1].double()).floor().long()
    last = (cum <= goal[:, None]).sum(1).clamp(max=vocab - 1)
    out = torch.where(i < kept[:, None], token, torch.where(i == kept[:, None], last[:, None], -1))
    return dict(tokens=out.to(torch.int32), count=(kept + 1).to(torch.int32))


# ---- one pass ------------------------------------------------------------------

def _own(s):
    c = s["case"]
    if c["op"] == "verify":
        from paper_2605_27255_gb300 import drafts
        tokens, count = drafts.verify(s["target"], s["drafted"], s["start"], s["u"], s["r"], draft=s["draft"],
                                      width=c["drafts"] + 1)
        return dict(tokens=tokens, count=count)
    from paper_2605_27255_gb300 import paged
    if c["op"] == "tables":
        if "tables" not in s:  # the object that a server keeps over its block table
            s["tables"] = paged.BlockTables(s["table"], s["held"], s["free"], s["n_free"])
        q_start, kv_len, slots, positions = s["tables"].advance(s["kept"], s["added"], s["tokens"])
        return dict(q_start=q_start, kv_len=kv_len, slots=slots, positions=positions, table=s["table"],
                    held=s["held"], free=s["free"], n_free=s["n_free"])
    if "cache" not in s:  # the handle that a server keeps over its pools
        s["cache"] = paged.PagedCache8(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], n_q=c["n_q"])
    if c["op"] == "append8":
        n_q, n_kv, x = c["n_q"], c["n_kv"], s["qkv"]
        q = s["cache"].append(x[:, :n_q], x[:, n_q:n_q + n_kv], x[:, n_q + n_kv:], s["q_start"], s["kv_len"],
                              q_gain=s["q_gain"], k_gain=s["k_gain"], eps=s["eps"], rope=s["rope"])
        return dict(q=q, k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return s["cache"].attend(s["q"], s["q_start"], s["kv_len"], scale=s["scale"], window=c["window"])


def run(state):
    if own:
        return _own(state)
    return {"tables": _plain_tables, "append8": _plain_append, "attend8": _plain_attend,
            "verify": _plain_verify}[state["case"]["op"]](state)


# ---- the definitions in 64 bits, sequence by sequence ----------------------------

def _exact_tables(s):
    np_ = lambda x: x.cpu().numpy().astype(np.int64)  # noqa: E731
    table, held, free, kept, added = map(np_, (s["table"], s["held"], s["free"], s["kept"], s["added"]))
    stack, width, room = list(free[:int(s["n_free"][0])]), table.shape[1], s["tokens"]
    asked = []
    for b in range(len(kept)):
        kept[b] = min(max(kept[b], 0), PAGE * held[b])
        first = _pages(kept[b])
        stack += list(table[b, first:held[b]])
        table[b, first:held[b]] = -1
        asked.append((first, _pages(kept[b] + added[b]) - first))
    free[:len(stack)] = stack
    sums, given = [0, 0], []
    for b, (first, want) in enumerate(asked):
        if first + want > width:
            given.append(False)
            continue
        sums = [sums[0] + want, sums[1] + added[b]]
        given.append((want == 0 or sums[0] <= len(stack)) and sums[1] <= room)
    left = len(stack) - sum(w for (_, w), g in zip(asked, given) if g)
    at, q_start, slots, positions = left, [0], [], []
    for b, ((first, want), g) in enumerate(zip(asked, given)):
        held[b] = first
        if not g:
            added[b] = 0
        else:
            table[b, first:first + want] = stack[at:at + want]
            at += want
            held[b] += want
        for p in range(kept[b], kept[b] + added[b]):
            positions.append(p)
            slots.append(table[b, p // PAGE] * PAGE + p % PAGE)
        q_start.append(q_start[-1] + added[b])
    pad = [-1] * (room - len(slots))
    out = dict(q_start=q_start, kv_len=kept + added, slots=slots + pad, positions=positions + pad, table=table,
               held=held, free=free, n_free=[left])
    return {k: torch.tensor(np.asarray(v), dtype=torch.int32, device=s["table"].device) for k, v in out.items()}


def _exact_verify(s):
    c, f8 = s["case"], torch.float64
    wide = c["drafts"] + 1
    start, drafted = s["start"].tolist(), s["drafted"].tolist()
    tokens, counts = [], []
    for b in range(c["batch"]):
        out, n = [], start[b + 1] - start[b]
        rest = None
        for i in range(n):
            p, t = s["target"][start[b] + b + i].to(f8), drafted[start[b] + i]
            q = torch.zeros_like(p) if s["draft"] is None else s["draft"][start[b] + i].to(f8)
            if s["draft"] is None:
                q[t] = 1
            if float(s["u"][start[b] + i]) * float(q[t]) >= float(p[t]):
                rest = (p - q).clamp(min=0)
                rest = rest if float(rest.sum()) > 0 else p
                break
            out.append(t)
        if rest is None:
            rest = s["target"][start[b + 1] + b].to(f8)
        cum = rest.cumsum(0)
        goal = float(s["r"][b]) * float(cum[-1])
        out.append(min(int(torch.searchsorted(cum, torch.tensor([goal], dtype=f8, device=cum.device), right=True)),
                       c["vocab"] - 1))
        counts.append(len(out))
        tokens.append(out + [-1] * (wide - len(out)))
    dev = s["u"].device
    return dict(tokens=torch.tensor(tokens, dtype=torch.int32, device=dev),
                count=torch.tensor(counts, dtype=torch.int32, device=dev))


def _exact_append(s):
    case = s["case"]
    past, new = _lengths(case)
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d_h"]
    f8, dev = torch.float64, s["k"].device
    table, starts = s["table"].tolist(), np.concatenate([[0], np.cumsum(new)])
    x = s["qkv"].to(f8)
    codes = [s["k"].to(f8), s["v"].to(f8)]
    scales = [s["k_scale"].to(f8), s["v_scale"].to(f8)]
    q = torch.zeros(x.shape[0], n_q, d, dtype=f8, device=dev)
    half = torch.arange(d // 2, device=dev, dtype=f8)
    for b, (p0, n) in enumerate(zip(past, new)):
        if not n:
            continue
        y = x[starts[b]:starts[b] + n]
        unit = lambda z, g: z / ((z ** 2).mean(-1, keepdim=True) + s["eps"]).sqrt() * g.to(f8)  # noqa: E731
        yq, yk = y[:, :n_q], y[:, n_q:n_q + n_kv]
        if case["norm"]:
            yq, yk = unit(yq, s["q_gain"]), unit(yk, s["k_gain"])
        pos = torch.arange(p0, p0 + n, device=dev)
        angle = torch.polar(torch.ones(n, d // 2, dtype=f8, device=dev),
                            pos.to(f8)[:, None] * 1.0e6 ** (-2 * half / d))[:, None]
        rot = lambda z: torch.view_as_real(  # noqa: E731
            torch.complex(z[..., :d // 2].contiguous(), z[..., d // 2:].contiguous()) * angle
        ).transpose(-1, -2).reshape(*z.shape)
        q[starts[b]:starts[b] + n] = rot(yq)
        for pool, scale, z in zip(codes, scales, (rot(yk), y[:, n_q + n_kv:])):
            for p in range(p0 // PAGE, (p0 + n - 1) // PAGE + 1):
                blk, lo = table[b][p], max(0, p0 - p * PAGE)
                part = z[max(0, p * PAGE - p0):(p + 1) * PAGE - p0].transpose(0, 1)  # [kv, entries, d]
                most = part.abs().amax((1, 2))
                want = 2.0 ** (torch.frexp(most.clamp(min=2.0 ** -300))[1] - 6).clamp(LOW, HIGH).to(f8)
                old = scale[blk].clone()
                now = torch.where((most > TOP * old) | (lo == 0), want, old)
                scale[blk] = now
                pool[blk, :, :lo] *= (old / now)[:, None, None]
                pool[blk, :, lo:lo + part.shape[1]] = part / now[:, None, None]
    return dict(q=q, k=codes[0], v=codes[1], k_scale=scales[0], v_scale=scales[1])


def _exact_attend(s):
    case, q, f8 = s["case"], s["q"].to(torch.float64), torch.float64
    past, new = _lengths(case)
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d_h"]
    grp, dev, w = n_q // n_kv, q.device, case["window"] or 1 << 40
    out = torch.zeros_like(q)
    at = 0
    for b, (p0, n) in enumerate(zip(past, new)):
        blk = s["table"][b].long()
        held = lambda x, y: (x.to(f8)[blk] * y.to(f8)[blk][..., None, None]).transpose(0, 1).reshape(n_kv, -1, d)  # noqa: E731
        kk, vv = held(s["k"], s["k_scale"]), held(s["v"], s["v_scale"])
        for i in range(0, n, 256):
            m = min(256, n - i)
            pos = torch.arange(p0 + i, p0 + i + m, device=dev)[:, None]
            lo, hi = max(0, p0 + i + 1 - w), p0 + i + m
            j = torch.arange(lo, hi, device=dev)
            hide = (j > pos) | (j <= pos - w)
            y = q[at + i:at + i + m].view(m, n_kv, grp, d).permute(1, 2, 0, 3)
            a = s["scale"] * y @ kk[:, None, lo:hi].transpose(2, 3)
            a = torch.softmax(a.masked_fill(hide, -math.inf), -1) @ vv[:, None, lo:hi]
            out[at + i:at + i + m] = a.permute(2, 0, 1, 3).reshape(m, n_q, d)
        at += n
    return out


def exact(case, seed):
    return {"tables": _exact_tables, "append8": _exact_append, "attend8": _exact_attend,
            "verify": _exact_verify}[case["op"]](prepare(case, seed))
