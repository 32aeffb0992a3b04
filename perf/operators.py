"""What the paged-cache operators are measured on.

Four operators of one attention layer over a paged key/value cache:

* ``append``  per-head RMSNorm of queries and keys, rotate-half position
              rotation, append of keys and values, page means of the keys;
* ``attend``  causal attention of ragged chunks of new tokens (one token up to
              thousands per sequence) over the cache, optionally windowed;
* ``scores``  the score of every visible page for every token and kv head,
              ``scale * sum over the group's heads of q . mean key of the page``;
* ``pages``   attention over the pages those scores select, with the selection.

A batch holds ``batch`` sequences; sequence b has ``n_b`` new tokens behind
``past_b`` cached entries (both follow from the case by ``_lengths``).  Head
shapes are the repository's models' (4b/9b: 32 query and 8 kv heads of 128,
bf16; tiny: 4 and 2 of 64, fp32; the cut-down fp32 model: 16 and 4 of 64) and
generic ones.  Blocks lie in a random order in a pool with spare blocks.

Values: keys and queries as a per-head norm leaves them (unit RMS times a gain
around one, some heads sharper), values N(0, 1).
"""
import math

import numpy as np
import torch

own = False

PAGE = 64
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, n_q, n_kv, d_h, dtype, batch, ctx, new, ragged, **kw):
    c = dict(name=name, op=op, n_q=n_q, n_kv=n_kv, d_h=d_h, dtype=dtype, batch=batch, ctx=ctx, new=new, ragged=ragged)
    c.update(kw)
    return c


def listed():
    return [
        # one user decoding: a token's heads from the fp32 projections into the cache (latency)
        _case("append-4b-b1", "append", 32, 8, 128, "bf16", 1, 1155, 1, False, in_f32=True, norm=True, means=False),
        # continuous batching: decoding sequences and prompts that join, page means kept for sparse reading
        _case("append-4b-b16-mixed", "append", 32, 8, 128, "bf16", 16, 1288, 300, True, in_f32=True, norm=True,
              means=True),
        # two long prompts at once, bf16 activations
        _case("append-4b-prompts", "append", 32, 8, 128, "bf16", 2, 0, 8191, False, in_f32=False, norm=True,
              means=True),
        # the smallest model, one user, fp32 (latency)
        _case("attend-tiny-b1", "attend", 4, 2, 64, "f32", 1, 51, 1, False, window=0),
        # a few users with long documents in their caches: the cache's bytes are the time
        _case("attend-4b-b4-long", "attend", 32, 8, 128, "bf16", 4, 15491, 1, False, window=0),
        # continuous batching: decoding sequences and prompt chunks in one call, all of different ages
        _case("attend-4b-b16-mixed", "attend", 32, 8, 128, "bf16", 16, 2415, 300, True, window=0),
        # the last chunk of a long prompt: the tensor cores' rate is the time
        _case("attend-4b-chunk", "attend", 32, 8, 128, "bf16", 1, 14336, 2048, False, window=0),
        # chunks of an fp32 model with a sliding window
        _case("attend-f32-window", "attend", 16, 4, 64, "f32", 6, 700, 129, True, window=256),
        # page scores of the long caches' decoding users
        _case("scores-4b-b4-long", "scores", 32, 8, 128, "bf16", 4, 15491, 1, False),
        # and of a chunk of a long prompt
        _case("scores-4b-chunk", "scores", 32, 8, 128, "bf16", 1, 15872, 512, False),
        # the long caches again, an eighth of their pages read
        _case("pages-4b-b4-long", "pages", 32, 8, 128, "bf16", 4, 15491, 1, False, top=32, sink=1, local=2),
        # a chunk of a long prompt, every token and kv head with pages of its own
        _case("pages-4b-chunk", "pages", 32, 8, 128, "bf16", 1, 15872, 512, False, top=16, sink=1, local=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 280)


def _plain_elements(case):
    """Elements of the largest array of the plain form."""
    past, new = _lengths(case)
    q, l = max(new), max(p + n for p, n in zip(past, new))
    if case["op"] == "attend":
        return case["batch"] * case["n_q"] * q * l
    if case["op"] == "pages":
        return sum(new) * case["n_kv"] * case["top"] * PAGE * case["d_h"]
    return 0


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "scores", "pages"])
    n_q, n_kv, d_h, dtype = rng.choice([(32, 8, 128, "bf16"), (32, 8, 128, "bf16"), (28, 4, 128, "bf16"),
                                        (16, 16, 64, "bf16"), (24, 2, 64, "bf16"), (8, 1, 128, "bf16"),
                                        (4, 2, 64, "f32"), (16, 4, 64, "f32"), (8, 8, 128, "f32")])
    f32 = dtype == "f32"
    batch = _log(rng, 1, 64)
    ctx = _log(rng, 16, 2048 if f32 else 16384)
    new = 1 if rng.random() < 0.4 else _log(rng, 2, 512 if f32 else 8191 if op == "append" else 2048)
    extra = {}
    if op == "append":
        extra = dict(in_f32=rng.random() < 0.5, norm=rng.random() < 0.75, means=rng.random() < 0.5)
    elif op == "attend":
        extra = dict(window=0 if rng.random() < 0.7 else _log(rng, 16, 4096))
    elif op == "pages":
        sink, local = rng.randint(0, 2), rng.randint(1, 3)
        extra = dict(top=max(sink + local, _log(rng, 4, 64)), sink=sink, local=local)
    c = _case("", op, n_q, n_kv, d_h, dtype, batch, ctx, new, rng.random() < 0.5, **extra)
    del c["name"]
    # no more than the operator's largest listed case (fp32 products run at a fraction of the bf16 rate)
    most = max(_cost(x) for x in listed() if x["op"] == op) / (16 if f32 else 1)
    while _cost(c) > most or _plain_elements(c) > 1_100_000_000:
        if c["batch"] > 1:
            c["batch"] = c["batch"] * 2 // 3
        elif c["new"] > 1:
            c["new"] = c["new"] * 2 // 3
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


def _visible(case):
    """Per new token: the entries it may attend to, as (first, last + 1)."""
    w = case.get("window", 0)
    for p, n in zip(*_lengths(case)):
        for i in range(n):
            yield max(0, p + i + 1 - w) if w else 0, p + i + 1


def work(case):
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d_h"]
    es = 4 if case["dtype"] == "f32" else 2
    past, new = _lengths(case)
    t = sum(new)
    if case["op"] == "append":
        ein = 4 if case["in_f32"] else 2
        by = t * (n_q + 2 * n_kv) * d * (ein + es) + t * d * 4
        if case["means"]:  # the earlier entries of a page that is continued, and the means
            by += sum((p % PAGE) * n_kv * d * es for p, n in zip(past, new) if n)
            by += sum((p + n - 1) // PAGE - p // PAGE + 1 for p, n in zip(past, new) if n) * n_kv * d * es
        return {"bytes": by, "flops": t * (n_q + n_kv) * d * 8}
    qo = 2 * t * n_q * d * es
    if case["op"] == "attend":
        w = case["window"]
        seen = sum(p + n - (max(0, p + 1 - w) if w else 0) for p, n in zip(past, new) if n)
        pairs = sum(b - a for a, b in _visible(case))
        return {"bytes": qo + 2 * seen * n_kv * d * es, "flops": 4 * d * n_q * pairs}
    pages = sum(-(-b // PAGE) for _, b in _visible(case))
    held = sum(-(-(p + n) // PAGE) for p, n in zip(past, new) if n)
    if case["op"] == "scores":
        row = -(-max(p + n for p, n in zip(past, new)) // PAGE)
        return {"bytes": t * n_q * d * es + held * n_kv * d * es + t * n_kv * row * 4,
                "flops": t * n_q * d + 2 * d * n_kv * pages}
    kept = sum(min(case["top"], -(-b // PAGE)) for _, b in _visible(case))
    return {"bytes": qo + pages * n_kv * 4 + t * n_kv * case["top"] * 4
            + 2 * min(kept, held) * PAGE * n_kv * d * es,
            "flops": 4 * d * n_q * kept * PAGE}


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    n_q, n_kv, d, dt = case["n_q"], case["n_kv"], case["d_h"], TYPES[case["dtype"]]
    past, new = _lengths(case)
    t = sum(new)
    most = max(p + n for p, n in zip(past, new))
    width = -(-most // PAGE)
    blocks = case["batch"] * width + 3
    randn = lambda *shape: torch.randn(*shape, generator=g, device=dev)  # noqa: E731
    sharp = (1.0 + 0.5 * (torch.arange(n_q, device=dev) % 3))[:, None]
    s = dict(case=case,
             k=randn(blocks, n_kv, PAGE, d).to(dt), v=randn(blocks, n_kv, PAGE, d).to(dt),
             table=torch.randperm(blocks, generator=g, device=dev)[:case["batch"] * width]
             .reshape(case["batch"], width).to(torch.int32),
             q_start=torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device=dev),
             kv_len=torch.tensor([p + n for p, n in zip(past, new)], dtype=torch.int32, device=dev),
             most_new=max(new), most_kv=most, scale=d ** -0.5)
    if case["op"] == "append":
        tin = torch.float32 if case["in_f32"] else torch.bfloat16
        # queries, keys and values as one projection leaves them: a row per token
        s["qkv"] = (randn(t, n_q + 2 * n_kv, d) * 2.0).to(tin)
        s["q_gain"] = (1 + 0.1 * randn(d)).to(dt) if case["norm"] else None
        s["k_gain"] = (1 + 0.1 * randn(d)).to(dt) if case["norm"] else None
        ang = torch.arange(width * PAGE, device=dev, dtype=torch.float64)[:, None] \
            * (1.0e6 ** (-torch.arange(0, d, 2, device=dev, dtype=torch.float64) / d))
        s["rope"] = torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()
        s["eps"] = 1e-6
        if case["means"]:
            s["means"] = s["k"].float().mean(2).to(dt)
        return s
    s["q"] = (randn(t, n_q, d) * sharp).to(dt)
    if case["op"] == "scores":
        s["means"] = s["k"].float().mean(2).to(dt)
    elif case["op"] == "pages":
        s["scores"] = randn(t, n_kv, width) * 1.5
        s["scores"][:, :, ::7] = 0.25  # equal scores too: the lower page goes first
    return s


# ---- the plain forms: elementary torch operations in 32 bits ------------------

def _tokens(s, t):
    """Sequence, index within it and position of every token."""
    at = torch.arange(t, device=s["k"].device)
    first = s["q_start"].long()
    b = torch.searchsorted(first[1:].contiguous(), at, right=True)
    i = at - first[b]
    return b, i, s["kv_len"].long()[b] - (first[b + 1] - first[b]) + i


def _plain_append(s):
    c, k, v = s["case"], s["k"], s["v"]
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
    page, slot = s["table"].long()[b, pos // PAGE], pos % PAGE
    k[page, :, slot] = turn(kn).to(k.dtype)
    v[page, :, slot] = vn.to(v.dtype)
    out = dict(q=turn(q).to(k.dtype), k=k, v=v)
    if c["means"]:
        blocks, width = k.shape[0], s["table"].shape[1]
        held = (s["kv_len"].long()[:, None] - PAGE * torch.arange(width, device=k.device)).clamp(0, PAGE)
        count = torch.zeros(blocks + 1, dtype=torch.long, device=k.device)
        count[torch.where(held > 0, s["table"].long(), blocks)] = held
        count = count[:blocks]
        live = torch.arange(PAGE, device=k.device) < count[:, None]
        mean = (k.float() * live[:, None, :, None]).sum(2) / count.clamp(min=1)[:, None, None]
        touched = torch.zeros(blocks, dtype=torch.bool, device=k.device)
        touched[page] = True
        s["means"].copy_(torch.where(touched[:, None, None], mean, s["means"].float()))
        out["means"] = s["means"]
    return out


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
    rows = lambda pool: pool[s["table"].long()].float().transpose(1, 2).reshape(nb, n_kv, -1, d)  # noqa: E731
    a = qp @ rows(s["k"]).transpose(2, 3) * s["scale"]
    pos = (s["kv_len"].long() - n)[:, None] + row
    j = torch.arange(a.shape[-1], device=q.device)
    see = j <= pos[..., None]
    if c["window"]:
        see &= j > pos[..., None] - c["window"]
    a = a.view(nb, n_kv, most, grp, -1).masked_fill_(~see[:, None, :, None], -math.inf)
    a = a.sub_(a.amax(-1, keepdim=True)).exp_()
    a = a.div_(a.sum(-1, keepdim=True))
    o = a.view(nb, n_kv, most * grp, -1) @ rows(s["v"])
    o = o.view(nb, n_kv, most, grp, d).transpose(1, 2)
    return o[b, i].reshape(t, c["n_q"], d).to(q.dtype)


def _plain_scores(s):
    c, q = s["case"], s["q"]
    t, width = q.shape[0], s["table"].shape[1]
    b, _, pos = _tokens(s, t)
    first = s["q_start"].long()
    most = s["most_new"]
    row = torch.arange(most, device=q.device)
    qs = q.float().view(t, c["n_kv"], -1, c["d_h"]).sum(2)
    qp = qs[(first[:-1, None] + row).clamp(max=t - 1)].transpose(1, 2)  # [b, kv, row, d]
    m = s["means"][s["table"].long()].float().permute(0, 2, 3, 1)       # [b, kv, d, page]
    sc = (qp @ m * s["scale"]).transpose(1, 2)[b, row_of(s, t)]
    return sc.masked_fill(torch.arange(width, device=q.device) > (pos // PAGE)[:, None, None], -math.inf)


def row_of(s, t):
    return _tokens(s, t)[1]


def _plain_select(s, pos):
    """Kept pages of every token and kv head, ascending, -1 behind them."""
    c, sc = s["case"], s["scores"]
    width = sc.shape[-1]
    p = torch.arange(width, device=sc.device)
    seen = (pos // PAGE + 1)[:, None, None]
    must = (p < c["sink"]) | (p >= seen - c["local"])
    key = sc.masked_fill(must, math.inf).masked_fill(p >= seen, -math.inf)
    top = min(c["top"], width)
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :top]
    best = best.masked_fill(torch.arange(top, device=sc.device) >= seen, width)
    best = best.masked_fill(best >= seen, width).sort(-1).values
    pages = torch.full((*sc.shape[:2], c["top"]), -1, dtype=torch.int32, device=sc.device)
    pages[..., :top] = best.masked_fill(best == width, -1).int()
    return pages


def _plain_pages(s):
    c, q = s["case"], s["q"]
    n_kv, d, t = c["n_kv"], c["d_h"], q.shape[0]
    b, _, pos = _tokens(s, t)
    pages = _plain_select(s, pos)
    at = pages.long().clamp(min=0)
    block = s["table"].long()[b[:, None, None], at]
    head = torch.arange(n_kv, device=q.device)[None, :, None]
    kk = s["k"][block, head].float().reshape(t, n_kv, -1, d)
    j = (at * PAGE)[..., None] + torch.arange(PAGE, device=q.device)
    see = ((pages >= 0)[..., None] & (j <= pos[:, None, None, None])).reshape(t, n_kv, 1, -1)
    a = q.float().view(t, n_kv, -1, d) @ kk.transpose(2, 3) * s["scale"]
    a = a.masked_fill(~see, -math.inf)
    a = (a - a.amax(-1, keepdim=True)).exp()
    a = a / a.sum(-1, keepdim=True)
    vv = s["v"][block, head].float().reshape(t, n_kv, -1, d)
    return dict(out=(a @ vv).reshape(t, c["n_q"], d).to(q.dtype), pages=pages)


# ---- one pass ------------------------------------------------------------------

def _cache(s):
    """The handle a serving program keeps over its pools and block table."""
    if "cache" not in s:
        from paper_2605_27255_gb300 import paged
        s["cache"] = paged.PagedCache(s["k"], s["v"], s["table"], n_q=s["case"]["n_q"], means=s.get("means"))
    return s["cache"]


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "scores": _plain_scores,
                "pages": _plain_pages}[op](s)
    cache = _cache(s)
    if op == "append":
        n_q, n_kv, x = c["n_q"], c["n_kv"], s["qkv"]
        q = cache.append(x[:, :n_q], x[:, n_q:n_q + n_kv], x[:, n_q + n_kv:], s["q_start"], s["kv_len"],
                         q_gain=s["q_gain"], k_gain=s["k_gain"], eps=s["eps"], rope=s["rope"])
        out = dict(q=q, k=s["k"], v=s["v"])
        if c["means"]:
            out["means"] = s["means"]
        return out
    if op == "attend":
        return cache.attend(s["q"], s["q_start"], s["kv_len"], scale=s["scale"], window=c["window"])
    if op == "scores":
        return cache.page_scores(s["q"], s["q_start"], s["kv_len"], scale=s["scale"])
    out, pages = cache.attend_pages(s["q"], s["scores"], s["q_start"], s["kv_len"], scale=s["scale"], top=c["top"],
                                    sink=c["sink"], local=c["local"])
    return dict(out=out, pages=pages)


# ---- the definitions in 64 bits, sequence by sequence ----------------------------

def exact(case, seed):
    s = prepare(case, seed)
    past, new = _lengths(case)
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d_h"]
    grp, dev = n_q // n_kv, s["k"].device
    table = s["table"].cpu().numpy()
    starts = np.concatenate([[0], np.cumsum(new)])
    f8 = torch.float64
    if case["op"] == "append":
        x = s["qkv"].to(f8)
        k, v, q = s["k"].to(f8), s["v"].to(f8), torch.zeros(x.shape[0], n_q, d, dtype=f8, device=dev)
        means = s["means"].to(f8) if case["means"] else None
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
            turn = torch.polar(torch.ones(n, d // 2, dtype=f8, device=dev),
                               pos.to(f8)[:, None] * 1.0e6 ** (-2 * half / d))[:, None]
            rot = lambda z: torch.view_as_real(  # noqa: E731
                torch.complex(z[..., :d // 2].contiguous(), z[..., d // 2:].contiguous()) * turn
            ).transpose(-1, -2).reshape(*z.shape)
            q[starts[b]:starts[b] + n] = rot(yq)
            blk = torch.from_numpy(table[b].astype(np.int64)).to(dev)
            k[blk[pos // PAGE], :, pos % PAGE] = rot(yk)
            v[blk[pos // PAGE], :, pos % PAGE] = y[:, n_q + n_kv:]
            if case["means"]:
                for p in range(p0 // PAGE, (p0 + n - 1) // PAGE + 1):
                    m = min(PAGE, p0 + n - p * PAGE)
                    means[table[b, p]] = k[table[b, p], :, :m].mean(1)
        out = dict(q=q, k=k, v=v)
        if case["means"]:
            out["means"] = means
        return out
    q = s["q"].to(f8)
    if case["op"] == "scores":
        out = torch.full((q.shape[0], n_kv, table.shape[1]), -math.inf, dtype=f8, device=dev)
        for b, (p0, n) in enumerate(zip(past, new)):
            for i in range(0, n, 64):
                m = min(64, n - i)
                width = (p0 + i + m - 1) // PAGE + 1
                mean = s["means"][torch.from_numpy(table[b, :width].astype(np.int64)).to(dev)].to(f8)
                qs = q[starts[b] + i:starts[b] + i + m].view(m, n_kv, grp, d)
                sc = s["scale"] * torch.einsum("tkgd,pkd->tkp", qs, mean)
                far = torch.arange(width, device=dev) * PAGE > torch.arange(p0 + i, p0 + i + m, device=dev)[:, None]
                out[starts[b] + i:starts[b] + i + m, :, :width] = sc.masked_fill(far[:, None], -math.inf)
        return out
    out = torch.zeros(q.shape[0], n_q, d, dtype=f8, device=dev)
    if case["op"] == "attend":
        w = case["window"] or 1 << 40
        for b, (p0, n) in enumerate(zip(past, new)):
            blk = torch.from_numpy(table[b].astype(np.int64)).to(dev)
            kk = s["k"][blk].to(f8).transpose(0, 1).reshape(n_kv, -1, d)
            vv = s["v"][blk].to(f8).transpose(0, 1).reshape(n_kv, -1, d)
            for i in range(0, n, 256):
                m = min(256, n - i)
                end = p0 + i + m
                pos = torch.arange(p0 + i, end, device=dev)[:, None]
                j = torch.arange(end, device=dev)
                hide = (j > pos) | (j <= pos - w)
                for h in range(n_q):
                    a = s["scale"] * q[starts[b] + i:starts[b] + i + m, h] @ kk[h // grp, :end].T
                    a = torch.softmax(a.masked_fill(hide, -math.inf), -1)
                    out[starts[b] + i:starts[b] + i + m, h] = a @ vv[h // grp, :end]
        return out
    t = q.shape[0]
    if t * n_kv > 20000:
        return None
    pages = np.full((t, n_kv, case["top"]), -1, np.int32)
    scores = s["scores"].cpu().numpy()
    for b, (p0, n) in enumerate(zip(past, new)):
        for i in range(n):
            tok, pos = starts[b] + i, p0 + i
            seen = pos // PAGE + 1
            fixed = {p for p in range(seen) if p < case["sink"] or p >= seen - case["local"]}
            for g in range(n_kv):
                rest = [p for p in np.argsort(-scores[tok, g, :seen], kind="stable") if p not in fixed]
                keep = sorted(list(fixed) + rest[:max(0, case["top"] - len(fixed))])
                pages[tok, g, :len(keep)] = keep
    for b, (p0, n) in enumerate(zip(past, new)):
        blk = torch.from_numpy(table[b].astype(np.int64)).to(dev)
        for i in range(n):
            tok, pos = starts[b] + i, p0 + i
            at = torch.from_numpy(pages[tok].astype(np.int64)).to(dev)  # [kv, top]
            kv = torch.arange(n_kv, device=dev)[:, None]
            kk = s["k"][blk[at.clamp(min=0)], kv].to(f8).reshape(n_kv, -1, d)
            vv = s["v"][blk[at.clamp(min=0)], kv].to(f8).reshape(n_kv, -1, d)
            j = (at[..., None] * PAGE + torch.arange(PAGE, device=dev))
            hide = ((at < 0)[..., None] | (j > pos)).reshape(n_kv, 1, -1)
            a = s["scale"] * q[tok].view(n_kv, grp, d) @ kk.transpose(1, 2)
            out[tok] = (torch.softmax(a.masked_fill(hide, -math.inf), -1) @ vv).reshape(n_q, d)
    return dict(out=out, pages=torch.from_numpy(pages).to(dev))
