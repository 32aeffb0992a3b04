"""The 8-bit cache's operators on the GPU against their definitions in 64 bits
(tests/paged_util.py, tests/paged8_util.py).

Tolerances of the attention, against the same codes and scales: the output's rounding is at most
half a bf16 step (2^-8 of a value); the weights that meet the values are rounded to fp16 (2^-11 of
a weight), and a weighted mean moves by no more than that times the largest value; everything else
is fp32 (2^-14 of the largest value holds its sums over thousands of entries).  In the 2-norm each
rounding has an rms of at most its half step / sqrt(3), and the weights' errors are independent:
2.3e-3 for the output, 0.3e-3 for the weights; 3e-3 holds both.

Codes: a stored value is the nearest code, so within half a step of it, 2^-4 of its magnitude or
2^-10 of the scale where it is subnormal; the fp32 norm and rotation before it move the value by a few 2^-22."""
import math

import pytest
import torch

from paged8_util import TOP, Batch8, put, scale_of
from paged_util import PAGE, Batch, ref_append, ref_attend
from paper_2605_27255_gb300 import capi, paged

pytestmark = pytest.mark.gpu


def check(got, ref, v_max):
    got = got.cpu().double()
    assert torch.isfinite(got).all()
    off = (got - ref).abs()
    assert (off <= 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2.0 ** -14) * v_max).all(), off.max()
    assert off.norm().item() <= 3e-3 * ref.norm().item() + 1e-12


def cache_of(x: Batch8):
    c = paged.PagedCache8(x.k8.cuda(), x.v8.cuda(), x.k_scale.cuda(), x.v_scale.cuda(), x.table.cuda(), n_q=x.x.n_q)
    return c, x.q_start.cuda(), x.kv_len.cuda()


def values_top(x: Batch8):
    return x.plain.v.nan_to_num(0.0).abs().max().item()


def run(x: Batch8, window=0, scale=None):
    c, qs, kl = cache_of(x)
    scale = scale or x.x.d_h ** -0.5
    got = c.attend(x.q.cuda(), qs, kl, window=window, scale=scale)
    check(got, ref_attend(x.plain, scale, window), values_top(x))
    capi.pipo_op_paged_check()


HEADS = [(4, 2, 64), (32, 8, 128), (7, 1, 128), (16, 1, 64), (3, 3, 128), (40, 8, 64), (20, 2, 128), (16, 1, 128)]
# entries (the new ones included) and new tokens of every sequence
SHAPES = {
    "one-entry": ([1], [1]),
    "one-token": ([52], [1]),
    "page-edges": ([63, 64, 65, 128, 129, 1], [1, 1, 1, 1, 1, 1]),
    "whole-prompt": ([193], [193]),
    "chunk": ([700], [131]),
    "ragged": ([300, 5, 64, 0, 515, 260], [1, 5, 64, 0, 70, 3]),
    "idle": ([100, 80, 70], [0, 2, 0]),
    "long": ([2500, 1900], [1, 2]),
    "drafts": ([640, 641, 130], [4, 4, 4]),
    "few": ([300, 17, 129], [9, 8, 7]),
    "middle": ([700, 90, 333, 0], [20, 30, 16, 0]),
    "middle-64": ([64, 128, 65, 1], [23, 22, 21, 1]),
}


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_attend_matches_float64(heads, shape):
    lens, new = SHAPES[shape]
    run(Batch8(lens, new, *heads, seed=len(shape)))


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [3, 1, 1, 9], [20, 1, 1, 60], [90, 1, 1, 300]])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 200, 100000, 2 ** 31 - 1])
def test_attend_window(d_h, new, window):
    run(Batch8([400, 70, 1, 300], new, 8, 2, d_h, seed=window % 1000), window)


@pytest.mark.parametrize("new", [[5, 2, 1], [60, 2, 1], [150, 2, 1]])
def test_tokens_without_an_entry_and_rows_of_no_sequence(new):
    """More new tokens than entries: zero outputs and nothing appended; rows
    outside every sequence stay as they were."""
    x = Batch8([3, 0, 130], new, 8, 2, 64, seed=3)
    c, qs, kl = cache_of(x)
    none, n = new[0] - 3, x.tokens
    out = torch.full((n + 4, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.cat([x.q, torch.full((4, 8, 64), float("nan"), dtype=torch.bfloat16)]).cuda()
    got = c.attend(q, qs, kl, out=out)
    assert (got[n:] == 7.0).all()
    assert (got[:none] == 0).all() and (got[none + 3:none + 5] == 0).all()
    check(got[:n], ref_attend(x.plain, 64 ** -0.5), values_top(x))
    before, scales = c.k.view(torch.uint8).clone(), c.k_scale.clone()
    k = torch.randn(n, 2, 64, device="cuda")
    y = torch.full((n, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    c.append(x.q.float().cuda(), k, k, qs, kl, out=y)
    assert (y[:none] == 0).all() and (y[none + 3:none + 5] == 0).all() and (y[none:none + 3] != 0).any()
    blk, last = x.table[0, 0].item(), x.table[2, 2].item()
    assert ((c.k[blk, :, :3].float() * c.k_scale[blk][:, None, None]).transpose(0, 1) -
            k[none:none + 3]).abs().max() <= 2.0 ** -4 * k.abs().max()
    same = torch.ones_like(before, dtype=torch.bool)
    same[blk, :, :3] = False
    same[last, :, 1] = False
    if (c.k_scale[last] != scales[last]).any():
        same[last] = False
    assert torch.equal(before[same], c.k.view(torch.uint8)[same])


@pytest.mark.parametrize("new", [[33, 1], [1, 1]])
def test_attend_strided_rows(new):
    """Queries as a slice of a fused row, outputs into a wider one."""
    x = Batch8([200, 77], new, 8, 2, 128, seed=8)
    c, qs, kl = cache_of(x)
    fused = torch.zeros(x.tokens, 12, 128, dtype=torch.bfloat16, device="cuda")
    fused[:, 2:10] = x.q.cuda()
    wide = torch.full((x.tokens, 10, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    c.attend(fused[:, 2:10], qs, kl, out=wide[:, 1:9])
    check(wide[:, 1:9], ref_attend(x.plain, 128 ** -0.5), values_top(x))
    assert (wide[:, 0] == 3).all() and (wide[:, 9] == 3).all()


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [7, 1, 3, 4], [30, 20, 10, 22], [7, 1, 130, 40], [200, 300, 5, 333]])
@pytest.mark.parametrize("window", [1, 50, 64, 200])
def test_attend_window_over_pages_that_are_gone(d_h, new, window):
    """What the window has passed for all of a sequence's new tokens may be NaN, codes and scales,
    and the table may hold anything for its pages."""
    x = Batch8([700, 333, 192, 1025], new, 8, 2, d_h, seed=13)
    ref = ref_attend(x.plain, d_h ** -0.5, window)
    top = values_top(x)
    for b in range(4):
        first = x.x.lens[b] - new[b] - window + 1
        for p in range(-(-x.x.lens[b] // PAGE)):
            gone, blk = min(PAGE, max(0, first - p * PAGE)), x.table[b, p].item()
            x.k8[blk, :, :gone] = float("nan")
            x.v8[blk, :, :gone] = float("nan")
            if gone == PAGE:
                x.k_scale[blk] = x.v_scale[blk] = float("nan")
                x.table[b, p] = -5 if p & 1 else 1 << 30
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl, window=window), ref, top)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("new", [[1, 1], [6, 5], [20, 18], [60, 200]])
def test_attend_blocks_of_different_scales(d_h, new):
    """Values of blocks that differ by up to 2^20, keys by up to 2^3: scales differ block by block."""
    run(Batch8([900, 650], new, 8, 2, d_h, seed=4, v_mult=(-18, 2), k_mult=(-2, 1)))


@pytest.mark.parametrize("new", [[1, 1], [6, 5], [20, 18], [60, 200]])
def test_attend_sharp_flat_and_tiny(new):
    """Queries of very different size in one tile: scores that single out one entry, or none."""
    x = Batch8([500, 333], new, 8, 2, 128, seed=6)
    size = 10.0 ** torch.linspace(-6, 1.5, x.tokens * 8).reshape(x.tokens, 8, 1)
    x.q = (x.q.float() * size).bfloat16()
    x.plain.q = x.q
    run(x)
    run(x, scale=1e-4)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("new", [[1, 1], [6, 5], [20, 18], [60, 200]])
def test_attend_every_code(d_h, new):
    """Pools of random bytes (all but NaN), subnormal codes among them, and blocks of subnormal codes alone."""
    x = Batch8([900, 650], new, 8, 2, d_h, seed=14)
    g = torch.Generator().manual_seed(15)
    for name, exps in (("k", (-9, -7)), ("v", (-12, 1))):
        raw = torch.randint(0, 256, x.k8.shape, generator=g, dtype=torch.uint8)
        raw[::3] &= 0x87
        raw[(raw & 0x7f) == 0x7f] = 0x7e
        scale = 2.0 ** torch.randint(exps[0], exps[1] + 1, x.k_scale.shape, generator=g).float()
        setattr(x, name + "8", raw.view(torch.float8_e4m3fn))
        setattr(x, name + "_scale", scale)
        setattr(x.plain, name, raw.view(torch.float8_e4m3fn).double() * scale[..., None, None].double())
    run(x)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("new", [[1, 1], [6, 5], [20, 18], [60, 200]])
def test_attend_any_scales(d_h, new):
    """Pools that were filled by something else: scales that are no powers of two, zeros in whole blocks, and keys
    and values far from one in size."""
    x = Batch8([900, 650], new, 8, 2, d_h, seed=18)
    g = torch.Generator().manual_seed(19)
    for name, size in (("k", 2.0 ** -30), ("v", 2.0 ** 40)):
        scale = getattr(x, name + "_scale") * size * (0.5 + torch.rand(x.k_scale.shape, generator=g))
        codes = getattr(x, name + "8")
        if name == "v":
            codes.view(torch.uint8)[x.table[0, 3].item()] = 0
        setattr(x, name + "_scale", scale)
        setattr(x.plain, name, codes.double() * scale[..., None, None].double())
    run(x, scale=2.0 ** 30 * d_h ** -0.5)


@pytest.mark.parametrize("new", [[1, 1], [6, 5], [20, 18], [60, 200]])
def test_attend_extreme_queries(new):
    """Rows of the smallest and of very large queries (equal weights, one entry's values), of zeros, and rows with
    an infinity or a NaN, which become NaN and leave the others alone."""
    x = Batch8([500, 333], new, 8, 2, 64, seed=16)
    size = torch.tensor([1e-39, 1e-37, 1e-34, 1e-20, 1e20, 1e28, 0.0, 1.0])[torch.arange(x.tokens * 8) * 5 % 8]
    x.q = (x.q.float() * size.reshape(x.tokens, 8, 1)).bfloat16()
    x.plain.q = x.q
    run(x)
    c, qs, kl = cache_of(x)
    want = c.attend(x.q.cuda(), qs, kl)
    odd = x.q.clone()
    odd[0, 3, 7], odd[-1, 4, 0] = float("inf"), float("nan")
    got = c.attend(odd.cuda(), qs, kl)
    assert got[0, 3].isnan().all() and got[-1, 4].isnan().all()
    got[0, 3], got[-1, 4] = want[0, 3], want[-1, 4]
    assert torch.equal(got, want)


def test_attend_long():
    run(Batch8([16000, 9000], [1, 1], 8, 2, 128, seed=31))


def test_attend_on_another_stream_and_in_a_graph():
    x = Batch8([600, 300, 80], [1, 1, 1], 32, 8, 128, seed=21)
    c, qs, kl = cache_of(x)
    q = x.q.cuda()
    eager = c.attend(q, qs, kl)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = c.attend(q, qs, kl)
    s.synchronize()
    assert torch.equal(eager, other)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = c.attend(q, qs, kl)
    kl -= torch.tensor([200, 0, 17], dtype=torch.int32, device="cuda")
    big = Batch8([4000] * 3, [100] * 3, 32, 8, 128, seed=22)
    cb, qsb, klb = cache_of(big)
    for _ in range(2):
        g.replay()
        cb.attend(big.q.cuda(), qsb, klb)
    torch.cuda.synchronize()
    x.plain.lens = [400, 300, 63]
    check(out, ref_attend(x.plain, 128 ** -0.5), values_top(x))


def test_attend_on_two_streams_and_in_two_graphs_at_once():
    """One object, calls that overlap: scratch is a stream's, or a graph's, own."""
    small, large = Batch8([900, 300], [1, 2], 32, 8, 128, seed=41), Batch8([900, 300], [300, 120], 32, 8, 128, seed=41)
    c, _, kl = cache_of(small)
    work = [(x.q.cuda(), x.q_start.cuda()) for x in (small, large)]
    want = [c.attend(q, qs, kl).clone() for q, qs in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [[], []]
    for _ in range(5):
        for i, (q, qs) in enumerate(work):
            with torch.cuda.stream(streams[i]):
                got[i].append(c.attend(q, qs, kl))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(want[i], y) for y in got[i])
    graphs, out = [], []
    for q, qs in work:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out.append(c.attend(q, qs, kl))
        graphs.append(g)
    for o in out:
        o.zero_()
    for _ in range(5):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.parametrize("new", [[1, 1, 1], [1, 40, 20], [1, 200, 70]])
def test_attend_empty_wide_and_clamped(new):
    """Sequences without entries, a table far wider than they need, lengths beyond it and below zero."""
    x = Batch8([130, 300, 64], new, 8, 2, 64, seed=42, width=5000)
    c, qs, kl = cache_of(x)
    q = x.q.cuda()
    check(c.attend(q, qs, kl), ref_attend(x.plain, 64 ** -0.5), values_top(x))
    for n in (0, -5, -2 ** 31):
        assert (c.attend(q, qs, torch.full_like(kl, n)) == 0).all()
    x = Batch8([128, 320, 64], new, 8, 2, 64, seed=43, width=5)
    c, qs, kl = cache_of(x)
    blocks = [t for row in x.table.tolist() for t in row if 0 <= t < x.x.blocks]
    c.table.copy_(torch.tensor((blocks * 5)[:15], dtype=torch.int32).reshape(3, 5))  # (every page is some block)
    top = torch.full_like(kl, 320)
    assert torch.equal(c.attend(q, qs, torch.full_like(kl, 2 ** 31 - 1)), c.attend(q, qs, top))


@pytest.mark.parametrize("new", [[1, 1, 3], [30, 1, 35], [200, 1, 64]])
def test_attend_same_inputs_same_bits(new):
    x = Batch8([1500, 300, 2000], new, 32, 8, 128, seed=9)
    c, qs, kl = cache_of(x)
    q = x.q.cuda()
    first = c.attend(q, qs, kl).clone()
    for _ in range(3):
        assert torch.equal(first, c.attend(q, qs, kl))


@pytest.mark.parametrize("new", [[1, 1, 3], [30, 1, 35], [200, 1, 64]])
def test_scratch_may_hold_anything(new):
    x = Batch8([1500, 300, 2000], new, 32, 8, 128, seed=9)
    c, qs, kl = cache_of(x)
    q = x.q.cuda()
    first = c.attend(q, qs, kl).clone()
    for fill in (0xff, 0x7f, 0):
        c._scratch.fill_(fill)
        assert torch.equal(first, c.attend(q, qs, kl))


def test_many_sequences():
    """The largest batch, mostly idle sequences."""
    n = 4096
    lens = [0] * n
    new = [0] * n
    for b in range(0, n, 97):
        lens[b], new[b] = 1 + b % 130, 1 + (b // 97) % min(3, 1 + b % 130)
    run(Batch8(lens, new, 4, 2, 64, seed=17))


@pytest.mark.parametrize("new", [1, 20, 40])
def test_blocks_past_32_bit_offsets(new):
    """Blocks whose entries lie more than 2^32 bytes into the pools."""
    x = Batch8([150], [new], 32, 8, 128, seed=40)
    blocks, first = 70000, 66000
    k8 = torch.zeros(blocks, 8, PAGE, 128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v8 = torch.zeros(blocks, 8, PAGE, 128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ks, vs = (torch.ones(blocks, 8, device="cuda") for _ in range(2))
    n = x.x.blocks
    for pool, src in ((k8.view(torch.uint8), x.k8.view(torch.uint8)), (v8.view(torch.uint8), x.v8.view(torch.uint8)),
                      (ks, x.k_scale), (vs, x.v_scale)):
        pool[first:first + n] = src.cuda()
    table = torch.where((x.table >= 0) & (x.table < n), x.table + first, x.table)
    c = paged.PagedCache8(k8, v8, ks, vs, table.cuda(), n_q=32)
    got = c.attend(x.q.cuda(), x.q_start.cuda(), x.kv_len.cuda())
    check(got, ref_attend(x.plain, 128 ** -0.5), values_top(x))
    k = torch.randn(new, 8, 128).bfloat16()
    c.append(None, k.cuda(), k.cuda(), x.q_start.cuda(), x.kv_len.cuda())
    blk = int(table[0, 149 // PAGE])
    got = c.k[blk, :, 149 % PAGE].float() * c.k_scale[blk][:, None]
    assert (got.cpu() - k[-1].float()).abs().max() <= 2.0 ** -4 * k.abs().max()


# ---- append

@pytest.mark.parametrize("tin", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS[:4])
@pytest.mark.parametrize("what", ["all", "rope", "norm", "plain"])
def test_append_matches_float64(tin, heads, what):
    n_q, n_kv, d_h = heads
    lens, new = [300, 5, 64, 0, 515, 260, 65], [1, 5, 64, 0, 70, 3, 2]
    x = Batch8(lens, new, n_q, n_kv, d_h, seed=len(what))
    c, qs, kl = cache_of(x)
    g = torch.Generator().manual_seed(77)
    qkv = (torch.randn(x.tokens, n_q + 2 * n_kv, d_h, generator=g) * 2).to(tin)
    gains = [(1 + 0.1 * torch.randn(d_h, generator=g)).bfloat16() for _ in range(2)] if what in ("all", "norm") else [None] * 2
    theta = 1e4 if what in ("all", "rope") else None
    rope = paged.rope_table(x.x.width * PAGE, d_h, theta) if theta else None
    dev = qkv.cuda()
    got = c.append(dev[:, :n_q], dev[:, n_q:n_q + n_kv], dev[:, n_q + n_kv:], qs, kl, rope=rope,
                   q_gain=None if gains[0] is None else gains[0].cuda(), k_gain=None if gains[1] is None else gains[1].cuda())
    rq, rk, rv = ref_append(x.x, qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:], *gains, 1e-6, theta)
    assert (got.cpu().double() - rq).abs().max() <= 2.0 ** -8 * 1.01 * rq.abs().max()
    for pool, scale, old8, old_scale, ref, exact in ((c.k, c.k_scale, x.k8, x.k_scale, rk, what == "plain"),
                                                     (c.v, c.v_scale, x.v8, x.v_scale, rv, True)):
        want, want_s = old8.double(), old_scale.double()
        at = 0
        for b, n in enumerate(new):
            if n:
                put(want, want_s, x.table[b], lens[b] - n, ref[at:at + n])
            at += n
        have, have_s = pool.cpu().double(), scale.cpu().double()
        assert torch.equal(have_s, want_s)
        if exact:  # inputs that reach the codes without a rounding
            assert torch.equal(have.nan_to_num(1e9), want.nan_to_num(1e9))
        else:
            at = 0
            for t, b, pos in x.x.each_token():
                blk = x.table[b, pos // PAGE].item()
                y, s = ref[t], have_s[blk][:, None]
                off = (have[blk, :, pos % PAGE] * s - y).abs()
                assert (off <= torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * s) * (1 + 2.0 ** -14)).all()
                want[blk, :, pos % PAGE] = have[blk, :, pos % PAGE]
            assert torch.equal(have.nan_to_num(1e9), want.nan_to_num(1e9))


def one(new_k, new_v, c, n, total, table_width=1):
    qs = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    kl = torch.tensor([total], dtype=torch.int32, device="cuda")
    c.append(None, new_k.cuda(), new_v.cuda(), qs, kl)


def empty_cache(blocks=2, n_kv=2, d_h=64):
    pool = lambda: torch.full((blocks, n_kv, PAGE, d_h), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
    junk = lambda: torch.full((blocks, n_kv), float("nan"), device="cuda")  # noqa: E731
    table = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
    return paged.PagedCache8(pool(), pool(), junk(), junk(), table, n_q=4)


@pytest.mark.parametrize("sizes", [[1e-3, 1.0, 300.0, 1e-6, 5e4], [0.0, 2.0, 0.0], [0.0, 0.0, 1e-30, 1e-3],
                                   [1e30, 1.0], [1e-38, 1e-20]])
def test_append_scales_follow_the_entries(sizes):
    """Token by token: the scale moves when an entry does not fit, codes held move with it."""
    c = empty_cache()
    g = torch.Generator().manual_seed(5)
    want, ws = torch.full((2, 2, PAGE, 64), float("nan"), dtype=torch.float64), torch.full((2, 2), float("nan"), dtype=torch.float64)
    for i, size in enumerate(sizes):
        x = (torch.randn(1, 2, 64, generator=g) * size)
        one(x, -x, c, 1, i + 1)
        put(want, ws, [0, 1], i, x.double())
        assert torch.equal(c.k_scale[0].cpu().double(), ws[0])
        assert torch.equal(c.k[0].cpu().double().nan_to_num(1e9), want[0].nan_to_num(1e9))
        assert torch.equal(c.v[0].cpu().double().nan_to_num(-1e9), -want[0].nan_to_num(1e9))
    assert (c.k_scale[1].isnan()).all()  # a block without entries is left alone


def test_append_not_finite():
    """Infinities saturate, NaN stays, and neither moves the scale of the others."""
    c = empty_cache()
    x = torch.ones(3, 2, 64)
    x[0, 0, 5], x[1, 0, 6], x[1, 1, 7] = float("inf"), float("-inf"), float("nan")
    one(x, x, c, 3, 3)
    assert (c.k_scale[0].cpu() == scale_of(1.0)).all()
    k = c.k[0, :, :3].cpu().float()
    assert k[0, 0, 5] == TOP and k[0, 1, 6] == -TOP and math.isnan(k[1, 1, 7])
    k[0, 0, 5] = k[0, 1, 6] = k[1, 1, 7] = 32.0
    assert (k == 32.0).all()


@pytest.mark.parametrize("cut", [[130], [64, 66], [1] * 130, [63, 1, 1, 65], [5, 100, 25]])
def test_append_cut_into_calls(cut):
    """However a prompt is cut: a stored value is within half a step of the entry, or (where the
    scale has grown over it) half a subnormal step more."""
    c = empty_cache(3, 2, 128)
    g = torch.Generator().manual_seed(6)
    x = torch.randn(130, 2, 128, generator=g) * torch.logspace(-4, 3, 130)[torch.randperm(130, generator=g)][:, None, None]
    at = 0
    for n in cut:
        one(x[at:at + n], x[at:at + n], c, n, at + n)
        at += n
    pos = torch.arange(130)
    for pool, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        s = scale.cpu().double()[pos // PAGE][..., None]
        got = pool.cpu().double()[pos // PAGE, :, pos % PAGE] * s
        off = (got - x.double()).abs()
        assert (off <= 2.0 ** -4 * x.abs() * (1 + 2.0 ** -4) + 2.0 ** -10 * s).all()


def test_append_without_queries_and_bad_blocks():
    x = Batch8([70, 10], [3, 2], 8, 2, 64, seed=2)
    c, qs, kl = cache_of(x)
    c.table[0, 1] = 1 << 29
    before = [t.clone() for t in (c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale)]
    k = torch.randn(5, 2, 64, device="cuda")
    assert c.append(None, k, k, qs, kl) is None
    blk = x.table[1, 0].item()
    for now, was in zip((c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale), before):
        other = torch.ones(x.x.blocks, dtype=torch.bool)
        other[blk] = False
        assert torch.equal(now.cpu()[other], was.cpu()[other])
    assert not torch.equal(c.k.view(torch.uint8)[blk], before[0][blk])


def test_append_in_a_graph_follows_the_lengths():
    c = empty_cache(4, 2, 64)
    qs = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    kl = torch.tensor([2], dtype=torch.int32, device="cuda")
    k = torch.zeros(2, 2, 64, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.append(None, k, k, qs, kl)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.append(None, k, k, qs, kl)
    gen = torch.Generator().manual_seed(8)
    want, ws = torch.full((4, 2, PAGE, 64), float("nan"), dtype=torch.float64), torch.ones(4, 2, dtype=torch.float64)
    for step in range(70):
        x = torch.randn(2, 2, 64, generator=gen) * (1 + step)
        k.copy_(x)
        kl.fill_(2 * step + 2)
        g.replay()
        put(want, ws, list(range(4)), 2 * step, x.double())
    got = c.k.cpu().double()
    assert torch.equal(got[:3].nan_to_num(1e9)[:, :, :12], want[:3].nan_to_num(1e9)[:, :, :12])
    assert torch.equal(c.k_scale.cpu().double()[:3], ws[:3])


def test_refusals():
    x = Batch8([70, 10], [3, 2], 8, 2, 64, seed=2)
    c, qs, kl = cache_of(x)
    q = x.q.cuda()
    with pytest.raises(ValueError):
        c.attend(q.float(), qs, kl)
    with pytest.raises(capi.PipoError):
        c.attend(q, qs, kl, window=-1)
    with pytest.raises(capi.PipoError):
        c.attend(q, qs, kl, scale=0.0)
    with pytest.raises(capi.PipoError):
        c.attend(q, qs, kl, scale=float("inf"))
    with pytest.raises(capi.PipoError, match="scratch"):
        capi.pipo_op_attn_paged8(c._c, 5, q.data_ptr(), 512, 0.1, 0, q.data_ptr(), 512, c.k.data_ptr(), 16)
    k = torch.zeros(5, 2, 64, device="cuda")
    with pytest.raises(capi.PipoError, match="rotations"):
        c.append(None, k, k, qs, kl, rope=paged.rope_table(64, 64, 1e4))
    with pytest.raises(ValueError):
        paged.PagedCache8(c.k.view(torch.uint8), c.v, c.k_scale, c.v_scale, c.table, n_q=8)
    with pytest.raises(ValueError):
        paged.PagedCache8(c.k, c.v, c.k_scale.double(), c.v_scale, c.table, n_q=8)
    with pytest.raises(ValueError):
        paged.PagedCache8(c.k, c.v, c.k_scale[:1], c.v_scale, c.table, n_q=8)
    for n_q in (7, 34, 0):  # no whole number of at most 16 per kv head
        with pytest.raises(capi.PipoError):
            paged.PagedCache8(c.k, c.v, c.k_scale, c.v_scale, c.table, n_q=n_q).attend(
                torch.zeros(5, n_q, 64, dtype=torch.bfloat16, device="cuda"), qs, kl)
    empty = torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    assert c.attend(empty, qs, kl).shape == (0, 8, 64)


def test_encode_is_what_append_stores():
    x = torch.randn(3, 2, PAGE, 64, device="cuda") * torch.tensor([1e-3, 1.0, 700.0], device="cuda")[:, None, None, None]
    codes, scale = paged.encode(x)
    c = empty_cache(3, 2, 64)
    one(x.transpose(1, 2).reshape(192, 2, 64), x.transpose(1, 2).reshape(192, 2, 64), c, 192, 192)
    assert torch.equal(c.k.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(c.k_scale, scale)
    assert torch.equal(c.v.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(c.v_scale, scale)
