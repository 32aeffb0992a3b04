"""The paged-cache operators on the GPU against their definitions in 64 bits
(tests/paged_util.py).

Tolerances.  fp32: products and sums of d_h = 128 terms and softmax weights in
fp32 carry a relative error of a few 2^-24 times the length of the longest
chain of additions; 2e-5 of the largest output holds them with room.  bf16:
outputs are rounded to 8 bits (2^-9 of a value at most), and the softmax
weights that meet the values on the tensor cores are too; a weighted mean of
values up to 4.5 with weight errors of 2^-9 each stays within 2^-9 * 4.5 on top
of half an ulp of the output: 2.5e-2 bounds both, and the error in the 2-norm
stays below 5e-3 (each rounding has an rms of about 2^-9 / sqrt(3))."""
import math

import pytest
import torch

from paged_util import PAGE, Batch, ref_append, ref_attend, ref_scores, ref_select
from paper_2605_27255_gb300 import capi, paged

pytestmark = pytest.mark.gpu

TOL = {torch.float32: (2e-5, 2e-6), torch.bfloat16: (2.5e-2, 5e-3)}  # (largest, 2-norm relative)


def check(got, ref, dtype):
    got = got.cpu().double()
    assert torch.isfinite(got).all()
    big, norm = TOL[dtype]
    scale = max(1.0, ref.abs().max().item())
    assert (got - ref).abs().max().item() <= big * scale
    n = ref.norm().item()
    assert (got - ref).norm().item() <= norm * n + 1e-12


def cache_of(x: Batch, means=None):
    c = paged.PagedCache(x.k.cuda(), x.v.cuda(), x.table.cuda(), n_q=x.n_q, means=means)
    return c, x.q_start.cuda(), x.kv_len.cuda()


HEADS = [(4, 2, 64), (32, 8, 128), (7, 1, 128), (16, 1, 64), (3, 3, 128), (40, 8, 64), (20, 2, 128)]
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
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS[:4])
@pytest.mark.parametrize("shape", sorted(SHAPES))
def test_attend_matches_float64(dtype, heads, shape):
    lens, new = SHAPES[shape]
    x = Batch(lens, new, *heads, dtype, seed=len(shape))
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl), ref_attend(x, heads[2] ** -0.5), dtype)
    capi.pipo_op_paged_check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS[4:])
def test_attend_other_head_groups(dtype, heads):
    x = Batch([333, 90, 7], [40, 1, 7], *heads, dtype, seed=5)
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl), ref_attend(x, heads[2] ** -0.5), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 200, 100000])
def test_attend_window(dtype, window):
    x = Batch([400, 70, 1, 300], [90, 1, 1, 300], 8, 2, 128, dtype, seed=window)
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl, window=window), ref_attend(x, 128 ** -0.5, window), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_without_an_entry_and_rows_of_no_sequence(dtype):
    """More new tokens than entries: zero outputs and nothing appended; rows
    outside every sequence stay as they were."""
    x = Batch([3, 0, 130], [5, 2, 1], 8, 2, 64, dtype, seed=3)
    c, qs, kl = cache_of(x)
    out = torch.full((x.tokens + 4, 8, 64), 7.0, dtype=dtype, device="cuda")
    q = torch.cat([x.q, torch.full((4, 8, 64), float("nan"), dtype=dtype)]).cuda()
    got = c.attend(q, qs, kl, out=out)
    assert (got[x.tokens:] == 7.0).all()
    assert (got[:2] == 0).all() and (got[5:7] == 0).all()
    check(got[:x.tokens], ref_attend(x, 64 ** -0.5), dtype)
    scores = torch.zeros(x.tokens + 4, 2, x.width, device="cuda")
    o2, pages = c.attend_pages(q, scores, qs, kl, top=4)
    assert (pages[:2] == -1).all() and (o2[:2] == 0).all()
    check(o2[:x.tokens], ref_attend(x, 64 ** -0.5), dtype)
    before = c.k.clone()
    k = torch.randn(x.tokens, 2, 64, device="cuda")
    y = torch.full((x.tokens, 8, 64), 7.0, dtype=dtype, device="cuda")
    c.append(x.q.float().cuda(), k, k, qs, kl, out=y)
    assert (y[:2] == 0).all() and (y[2:5] != 0).any()
    blk = x.table[0, 0].item()
    assert torch.equal(c.k[blk, :, :3].transpose(0, 1), k[2:5].to(dtype))
    same = torch.ones_like(before, dtype=torch.bool)
    same[blk, :, :3] = False
    same[x.table[2, 2].item(), :, 1] = False
    assert torch.equal(before.nan_to_num()[same], c.k.nan_to_num()[same])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_strided_rows(dtype):
    """Queries as a slice of a fused row, outputs into a wider one."""
    x = Batch([200, 77], [33, 1], 8, 2, 128, dtype, seed=8)
    c, qs, kl = cache_of(x)
    fused = torch.zeros(x.tokens, 12, 128, dtype=dtype, device="cuda")
    fused[:, 2:10] = x.q.cuda()
    wide = torch.full((x.tokens, 10, 128), 3.0, dtype=dtype, device="cuda")
    c.attend(fused[:, 2:10], qs, kl, out=wide[:, 1:9])
    check(wide[:, 1:9], ref_attend(x, 128 ** -0.5), dtype)
    assert (wide[:, 0] == 3).all() and (wide[:, 9] == 3).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [7, 1, 130, 40], [200, 300, 5, 333]])
@pytest.mark.parametrize("window", [1, 50, 64, 200])
def test_attend_window_over_pages_that_are_gone(dtype, d_h, new, window):
    """What the window has passed for all of a sequence's new tokens may be NaN,
    and the table may hold anything for its pages."""
    x = Batch([700, 333, 192, 1025], new, 8, 2, d_h, dtype, seed=13)
    ref = ref_attend(x, d_h ** -0.5, window)
    for b in range(4):
        first = x.lens[b] - new[b] - window + 1
        for p in range(-(-x.lens[b] // PAGE)):
            gone = min(PAGE, max(0, first - p * PAGE))
            x.k[x.table[b, p].item(), :, :gone] = float("nan")
            x.v[x.table[b, p].item(), :, :gone] = float("nan")
            if gone == PAGE:
                x.table[b, p] = -5 if p & 1 else 1 << 30
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl, window=window), ref, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_sharp_and_flat_scores(dtype):
    """Scores of a hundred and more (one entry takes all the weight) and all equal."""
    x = Batch([500], [3], 4, 2, 64, dtype, seed=1)
    x.q = x.q * 40
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl), ref_attend(x, 0.125), dtype)
    x.q.zero_()
    check(c.attend(x.q.cuda(), qs, kl), ref_attend(x, 0.125), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_rising_scores(dtype):
    """The running maximum moves in every tile, by little and by much."""
    for step in (0.02, 1.0):
        x = Batch([600], [40], 4, 2, 64, dtype, seed=2)
        for p in range(10):
            blk = x.table[0, p].item()
            for s in range(PAGE):
                j = p * PAGE + s
                if j < 600:
                    x.k[blk, :, s] = 0.0
                    x.k[blk, :, s, 0] = j * step
        x.q.zero_()
        x.q[:, :, 0] = 1.0
        c, qs, kl = cache_of(x)
        check(c.attend(x.q.cuda(), qs, kl, scale=1.0), ref_attend(x, 1.0), dtype)


def test_attend_on_another_stream_and_in_a_graph():
    """Calls run on the current stream; a captured call follows lengths that grow."""
    x = Batch([900, 130], [1, 1], 32, 8, 128, torch.bfloat16, seed=4)
    c, qs, kl = cache_of(x)
    q = x.q.cuda()
    ref = ref_attend(x, 128 ** -0.5)
    c.attend(q, qs, kl)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out = c.attend(q, qs, kl)
    s.synchronize()
    check(out, ref, torch.bfloat16)
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attend(q, qs, kl, out=out)
    shorter = Batch([900, 130], [1, 1], 32, 8, 128, torch.bfloat16, seed=4)
    shorter.lens = [411, 65]
    kl.copy_(torch.tensor(shorter.lens, dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    check(out, ref_attend(shorter, 128 ** -0.5), torch.bfloat16)


def test_attend_same_inputs_same_bits():
    x = Batch([3000, 40, 700], [1, 40, 200], 32, 8, 128, torch.bfloat16, seed=6)
    c, qs, kl = cache_of(x)
    a = c.attend(x.q.cuda(), qs, kl)
    b = c.attend(x.q.cuda(), qs, kl)
    assert torch.equal(a, b)


# ---- append ----------------------------------------------------------------------

@pytest.mark.parametrize("tin", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS[:4])
@pytest.mark.parametrize("what", ["all", "rope", "norm", "plain"])
def test_append_matches_float64(tin, dtype, heads, what):
    n_q, n_kv, d = heads
    x = Batch([130, 1, 64, 70, 0, 300], [66, 1, 1, 5, 0, 300], n_q, n_kv, d, dtype, seed=9)
    means = torch.full((x.blocks, n_kv, d), 5.0, dtype=dtype, device="cuda")
    c, qs, kl = cache_of(x, means)
    g = torch.Generator().manual_seed(3)
    qkv = (3 * torch.randn(x.tokens, n_q + 2 * n_kv, d, generator=g)).to(tin)
    q, k, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
    gains = [(1 + 0.1 * torch.randn(d, generator=g)).to(dtype) for _ in range(2)] if what in ("all", "norm") else [None] * 2
    theta = 1.0e4 if what in ("all", "rope") else None
    rope = paged.rope_table(x.width * PAGE, d, theta) if theta else None
    k0, v0 = c.k.clone(), c.v.clone()
    dev = qkv.cuda()
    got = c.append(dev[:, :n_q], dev[:, n_q:n_q + n_kv], dev[:, n_q + n_kv:], qs, kl,
                   q_gain=None if gains[0] is None else gains[0].cuda(),
                   k_gain=None if gains[1] is None else gains[1].cuda(), rope=rope)
    rq, rk, rv = ref_append(x, q, k, v, gains[0], gains[1], 1e-6, theta)
    # one rounding to the pools' type of values computed in fp32 (the fp32 angles' table: 2^-24 of a value)
    tol = 2.0 ** -8 if dtype == torch.bfloat16 else 2e-6
    assert ((got.cpu().double() - rq).abs() <= tol * rq.abs() + tol * 1e-3 + (0 if dtype == torch.bfloat16 else 2e-6)
            + 2e-6 * rq.abs().max()).all()
    kd, vd = c.k.cpu(), c.v.cpu()
    written = torch.zeros(x.blocks, PAGE, dtype=torch.bool)
    for t, b, pos in x.each_token():
        blk, slot = x.table[b, pos // PAGE].item(), pos % PAGE
        written[blk, slot] = True
        assert ((kd[blk, :, slot].double() - rk[t]).abs() <= tol * rk[t].abs() + 2e-6 * rk.abs().max()).all()
        assert torch.equal(vd[blk, :, slot], v[t].to(dtype))
    keep = ~written[:, None, :].expand(-1, n_kv, -1)
    assert torch.equal(kd[keep].nan_to_num(), k0.cpu()[keep].nan_to_num())
    assert torch.equal(vd[keep].nan_to_num(), v0.cpu()[keep].nan_to_num())
    # the means of the pages that received entries, of the keys as stored
    touched = set()
    for _, b, pos in x.each_token():
        touched.add((b, pos // PAGE))
    md = means.cpu().double()
    for b, p in touched:
        blk = x.table[b, p].item()
        m = min(PAGE, x.lens[b] - p * PAGE)
        ref = kd[blk, :, :m].double().mean(1)
        assert ((md[blk] - ref).abs() <= (2.0 ** -8 if dtype == torch.bfloat16 else 1e-6) * ref.abs() + 2e-6).all()
    others = [i for i in range(x.blocks) if i not in {x.table[b, p].item() for b, p in touched}]
    assert (means[others] == 5.0).all()


def test_append_without_queries_and_bad_blocks():
    """Keys and values alone; a block outside the pool is not followed."""
    x = Batch([10, 20], [10, 3], 8, 2, 64, torch.bfloat16, seed=2)
    x.table[1, 0] = -5
    c, qs, kl = cache_of(x)
    before = c.k.clone()
    k = torch.randn(x.tokens, 2, 64, device="cuda")
    assert c.append(None, k, k, qs, kl) is None
    blk = x.table[0, 0].item()
    assert torch.equal(c.k[blk, :, :10].transpose(0, 1), k[:10].to(torch.bfloat16))
    assert torch.equal(c.k[blk, :, 10:].nan_to_num(), before[blk, :, 10:].nan_to_num())
    rest = [i for i in range(x.blocks) if i != blk]
    assert torch.equal(c.k[rest].nan_to_num(), before[rest].nan_to_num())


# ---- page scores and selection ------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", HEADS[:4])
@pytest.mark.parametrize("shape", ["one-entry", "page-edges", "chunk", "ragged", "long"])
def test_page_scores_match_float64(dtype, heads, shape):
    lens, new = SHAPES[shape]
    x = Batch(lens, new, *heads, dtype, seed=21, width=(max(lens) + PAGE - 1) // PAGE + 1)
    g = torch.Generator().manual_seed(2)
    means = torch.randn(x.blocks, heads[1], heads[2], generator=g).to(dtype)
    c, qs, kl = cache_of(x, means.cuda())
    got = c.page_scores(x.q.cuda(), qs, kl, scale=0.25).cpu().double()
    ref = ref_scores(x, means, 0.25)
    assert torch.equal(torch.isinf(got), torch.isinf(ref)) and not torch.isnan(got).any()
    fin = torch.isfinite(ref)
    # fp32 sums of up to 16 x 128 products of magnitude about 2: 2e-5 of the largest
    assert (got[fin] - ref[fin]).abs().max() <= 2e-5 * max(1.0, ref[fin].abs().max().item())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top,sink,local", [(1, 0, 0), (1, 0, 1), (3, 1, 2), (7, 2, 1), (16, 0, 1), (64, 1, 1)])
@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128), (7, 1, 128)])
def test_attend_pages(dtype, top, sink, local, heads):
    lens, new = [1500, 64, 65, 0, 900, 1], [2, 1, 1, 0, 37, 1]
    x = Batch(lens, new, *heads, dtype, seed=top)
    c, qs, kl = cache_of(x)
    g = torch.Generator().manual_seed(top)
    sc = torch.randn(x.tokens, heads[1], x.width, generator=g)
    sc[:, :, 2::5] = 0.5       # ties
    sc[0, :, 4] = float("nan")
    sc[1, :, 3] = float("inf")
    sc[2, :, :] = float("-inf")
    sc[5, :, 1::2] = -0.0
    sc[5, :, 0::2] = 0.0
    out, pages = c.attend_pages(x.q.cuda(), sc.cuda(), qs, kl, top=top, sink=sink, local=local)
    ref = ref_select(x, sc, top, sink, local)
    assert torch.equal(pages.cpu(), ref)
    check(out, ref_attend(x, heads[2] ** -0.5, pages=ref), dtype)
    capi.pipo_op_paged_check()


def test_attend_pages_of_everything_is_attend():
    x = Batch([777, 200], [1, 65], 32, 8, 128, torch.bfloat16, seed=13)
    c, qs, kl = cache_of(x)
    sc = torch.zeros(x.tokens, 8, x.width, device="cuda")
    out, _ = c.attend_pages(x.q.cuda(), sc, qs, kl, top=x.width, sink=0, local=1)
    check(out, ref_attend(x, 128 ** -0.5), torch.bfloat16)


# ---- refusals -------------------------------------------------------------------------

def test_refusals():
    x = Batch([100], [2], 8, 2, 64, torch.bfloat16, seed=1)
    c, qs, kl = cache_of(x)
    q = x.q.cuda()

    def refused(call):
        with pytest.raises(capi.PipoError) as e:
            call()
        assert e.value.status == capi.PIPO_EINVAL

    refused(lambda: c.attend(q, qs, kl, scale=0.0))
    refused(lambda: c.attend(q, qs, kl, scale=float("nan")))
    refused(lambda: c.attend(q, qs, kl, window=-1))
    refused(lambda: c.attend_pages(q, torch.zeros(2, 2, x.width, device="cuda"), qs, kl, top=1, sink=1, local=1))
    k = torch.zeros(2, 2, 64, device="cuda")
    refused(lambda: c.append(None, k, k, qs, kl, rope=paged.rope_table(16, 64, 1e4)))
    refused(lambda: c.append(None, k, k, qs, kl, eps=float("nan")))
    for bad in (lambda: c.attend(q.float(), qs, kl), lambda: c.attend(q, qs.long(), kl),
                lambda: c.attend(q[:, :4], qs, kl), lambda: c.page_scores(q, qs, kl),
                lambda: c.attend_pages(q, torch.zeros(2, 2, x.width + 1, device="cuda"), qs, kl, top=2),
                lambda: paged.PagedCache(c.k, c.v[:1], c.table, n_q=8),
                lambda: paged.PagedCache(c.k, c.v, c.table.long(), n_q=8)):
        with pytest.raises(ValueError):
            bad()
    w = torch.empty(64, dtype=torch.uint8, device="cuda")
    c._c.n_q_heads = 7  # not a multiple of the kv heads
    assert capi.pipo_op_attn_paged_scratch(c._c, 2) == 0
    refused(lambda: capi.pipo_op_attn_paged(c._c, 2, q.data_ptr(), 512, 0.1, 0, q.data_ptr(), 512, w.data_ptr(), 64))
    c._c.n_q_heads = 8
    need = capi.pipo_op_attn_paged_scratch(c._c, 2)
    refused(lambda: capi.pipo_op_attn_paged(c._c, 2, q.data_ptr() + 2, 512, 0.1, 0, q.data_ptr(), 512, w.data_ptr(), need))
    refused(lambda: capi.pipo_op_attn_paged(c._c, 2, q.data_ptr(), 511, 0.1, 0, q.data_ptr(), 512, w.data_ptr(), need))
    refused(lambda: capi.pipo_op_attn_paged(c._c, 2, q.data_ptr(), 512, 0.1, 0, q.data_ptr(), 512, w.data_ptr(), need - 1))
    refused(lambda: capi.pipo_op_attn_paged(c._c, 2, q.data_ptr(), 512, 0.1, 0, 0, 512, w.data_ptr(), need))


def test_nothing_to_do_is_a_no_op():
    x = Batch([100], [0], 8, 2, 64, torch.bfloat16, seed=1)
    c, qs, kl = cache_of(x)
    assert c.attend(x.q.cuda(), qs, kl).shape == (0, 8, 64)
    k = torch.zeros(0, 2, 64, device="cuda")
    before = c.k.clone()
    c.append(None, k, k, qs, kl)
    assert torch.equal(c.k.nan_to_num(), before.nan_to_num())


@pytest.mark.parametrize("top,sink,local", [(4, 1, 1), (6, 0, 0), (20, 2, 3)])
@pytest.mark.parametrize("heads", [(8, 2, 64), (32, 8, 128), (7, 1, 128), (16, 16, 64)])
def test_attend_pages_of_chunks(top, sink, local, heads):
    """Chunks long enough that whole tiles of tokens read each page once and
    mask by the selection."""
    lens, new = [1100, 300, 0, 70, 2200], [200, 300, 0, 1, 140]
    x = Batch(lens, new, *heads, torch.bfloat16, seed=top)
    c, qs, kl = cache_of(x)
    g = torch.Generator().manual_seed(top)
    sc = torch.randn(x.tokens, heads[1], x.width, generator=g)
    sc[:, :, 2::5] = 0.5
    sc[3] = float("-inf")
    sc[7] = float("nan")
    out, pages = c.attend_pages(x.q.cuda(), sc.cuda(), qs, kl, top=top, sink=sink, local=local)
    ref = ref_select(x, sc, top, sink, local)
    assert torch.equal(pages.cpu(), ref)
    check(out, ref_attend(x, heads[2] ** -0.5, pages=ref), torch.bfloat16)
    capi.pipo_op_paged_check()


def test_example_serves_requests_together_and_alone():
    """examples/paged_layer.py: the four operators between the projections.  A
    request's outputs do not depend on what shares its batch beyond the
    roundings to bf16 (queries, keys, weights and outputs, 2^-9 of a value
    each, against sums in another order), and all pages selected are dense
    attention."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_layer.py")
    spec = importlib.util.spec_from_file_location("paged_layer", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    layer = ex.Layer()
    g = torch.Generator(device="cuda").manual_seed(3)
    inputs = [torch.randn(n, layer.hidden, generator=g, device="cuda") for n in (400, 1, 150)]
    mixed = ex.serve(layer, inputs)
    for x, y, every in zip(inputs, mixed, ex.serve(layer, inputs, top=64)):
        alone = ex.serve(layer, [x])[0]
        assert torch.isfinite(y).all()
        assert (y - alone).norm() <= 2e-2 * alone.norm()
        assert (y - every).norm() <= 2e-2 * alone.norm()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_blocks_past_32_bit_offsets(dtype):
    """Blocks whose elements lie past 2^31 of the pool."""
    x = Batch([200, 70, 1], [70, 1, 1], 32, 8, 128, dtype, seed=3)
    high = 36000 - x.blocks  # 36000 blocks of 8 x 64 x 128 elements: 2.36e9
    assert high * 8 * 64 * 128 > 2 ** 31
    pools = []
    for pool in (x.k, x.v):
        p = torch.empty(36000, 8, 64, 128, dtype=dtype, device="cuda")
        p[high:] = pool.cuda()
        pools.append(p)
    table = torch.where(x.table < x.blocks, x.table + high, x.table)
    means = torch.zeros(36000, 8, 128, dtype=dtype, device="cuda")
    c = paged.PagedCache(*pools, table.cuda(), n_q=32, means=means)
    qs, kl = x.q_start.cuda(), x.kv_len.cuda()
    ref = ref_attend(x, 128 ** -0.5)
    check(c.attend(x.q.cuda(), qs, kl), ref, dtype)
    out, _ = c.attend_pages(x.q.cuda(), torch.zeros(x.tokens, 8, x.width, device="cuda"), qs, kl, top=x.width)
    check(out, ref, dtype)
    k = torch.randn(x.tokens, 8, 128, device="cuda")
    c.append(None, k, k, qs, kl)
    for t, b, pos in x.each_token():
        blk = table[b, pos // PAGE].item()
        assert torch.equal(c.k[blk, :, pos % PAGE], k[t].to(dtype)) and torch.equal(c.v[blk, :, pos % PAGE], k[t].to(dtype))
    assert (means[table[1, 1].item()] != 0).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scratch_may_hold_anything(dtype):
    x = Batch([900, 40, 700, 0], [1, 40, 200, 0], 32, 8, 128, dtype, seed=6)
    c, qs, kl = cache_of(x)
    a = c.attend(x.q.cuda(), qs, kl).clone()
    sc = torch.randn(x.tokens, 8, x.width, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    b = c.attend_pages(x.q.cuda(), sc, qs, kl, top=5)[0].clone()
    for junk in (0, 255, 1, 127):
        c._scratch.fill_(junk)
        assert torch.equal(c.attend(x.q.cuda(), qs, kl), a)
        c._scratch.fill_(junk)
        assert torch.equal(c.attend_pages(x.q.cuda(), sc, qs, kl, top=5)[0], b)


def test_many_sequences():
    """More sequences than a block has threads, most of them idle or short."""
    n = 1500
    lens = [(b * 37) % 150 for b in range(n)]
    new = [0 if b % 5 else min(1 + b % 3, max(1, lens[b])) for b in range(n)]
    for dtype in (torch.bfloat16, torch.float32):
        x = Batch(lens, new, 4, 2, 64, dtype, seed=1)
        means = torch.randn(x.blocks, 2, 64, generator=torch.Generator().manual_seed(1)).to(dtype)
        c, qs, kl = cache_of(x, means.cuda())
        check(c.attend(x.q.cuda(), qs, kl), ref_attend(x, 0.125), dtype)
        got, ref = c.page_scores(x.q.cuda(), qs, kl).cpu().double(), ref_scores(x, means, 0.125)
        fin = torch.isfinite(ref)
        assert torch.equal(fin, torch.isfinite(got)) and (got[fin] - ref[fin]).abs().max() <= 2e-5 * ref[fin].abs().max()
        k = torch.randn(x.tokens, 2, 64, device="cuda")
        c.append(None, k, k, qs, kl)
        for t, b, pos in x.each_token():
            if pos >= 0:
                assert torch.equal(c.k[x.table[b, pos // PAGE].item(), :, pos % PAGE], k[t].to(dtype))


def test_a_graph_keeps_its_scratch_beside_larger_calls():
    """A captured decode step is replayed after a long chunk has gone through the same object:
    its replays write nothing that other tensors own by then, and their outputs stay right."""
    x = Batch([5000, 130], [1, 1], 32, 8, 128, torch.bfloat16, seed=4)
    c, qs, kl = cache_of(x)
    q, ref = x.q.cuda(), ref_attend(x, 128 ** -0.5)
    sc = torch.zeros(2, 8, x.width, device="cuda")
    c.attend(q, qs, kl)
    g, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(g):
        c.attend(q, qs, kl, out=out)
        some = c.attend_pages(q, sc, qs, kl, top=x.width)[0]
    chunk = Batch([5000, 130], [2000, 100], 32, 8, 128, torch.bfloat16, seed=4)
    c.attend(chunk.q.cuda(), chunk.q_start.cuda(), kl)
    other = [torch.full((n << 20,), 7, dtype=torch.uint8, device="cuda") for n in (1, 2, 4, 8, 16, 32, 64)]
    for _ in range(3):
        out.zero_()
        g.replay()
        c.attend(chunk.q.cuda(), chunk.q_start.cuda(), kl)
        torch.cuda.synchronize()
        check(out, ref, torch.bfloat16)
        check(some, ref, torch.bfloat16)
    assert all((t == 7).all() for t in other)


@pytest.mark.parametrize("tin", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_queries_without_an_entry_are_zero_with_norms(tin, dtype, d_h, eps):
    """A token with a negative position has zero queries, whatever the norm makes of nothing."""
    x = Batch([3, 0, 130], [5, 2, 1], 8, 2, d_h, dtype, seed=3)
    c, qs, kl = cache_of(x)
    g = torch.Generator().manual_seed(3)
    q, k = (torch.randn(x.tokens, n, d_h, generator=g).to(tin).cuda() for n in (8, 2))
    gain = torch.ones(d_h, dtype=dtype, device="cuda")
    y = c.append(q, k, k, qs, kl, q_gain=gain, k_gain=gain, eps=eps, rope=paged.rope_table(x.width * PAGE, d_h, 1e4))
    assert (y[:2] == 0).all() and (y[5:7] == 0).all()
    assert torch.isfinite(y).all() and (y[2:5] != 0).any() and (y[7] != 0).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 70, 2 ** 30, 449, 448, 447])
def test_attend_windows_of_every_entry(dtype, window):
    """A window longer than any sequence hides nothing, also where more tokens than entries put
    positions below zero; so do windows of and just below the longest sequence's 448 entries."""
    x = Batch([5, 70, 0, 448, 130], [10, 150, 2, 448, 1], 8, 2, 64, dtype, seed=3)
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl, window=window), ref_attend(x, 0.125, window), dtype)


# ---- long tables: more than one block of pages per score row, every width of the selection ------
# (tolerances as above: scores are within a few 2^-24 of their size, which moves a weight by 1e-6 at
# most, whatever the number of entries)

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [[1, 1], [1, 45], [0, 3]])
@pytest.mark.parametrize("lens,width", [([4160, 8200], 0), ([4096, 4097], 0), ([130, 9000], 300)])
def test_page_scores_of_many_pages(dtype, new, lens, width):
    x = Batch(lens, new, 6, 2, 64, dtype, seed=3, width=width or None)
    means = torch.randn(x.blocks, 2, 64, generator=torch.Generator().manual_seed(2)).to(dtype)
    c, qs, kl = cache_of(x, means.cuda())
    got, ref = c.page_scores(x.q.cuda(), qs, kl, scale=0.25).cpu().double(), ref_scores(x, means, 0.25)
    assert torch.equal(torch.isinf(got), torch.isinf(ref)) and not torch.isnan(got).any()
    fin = torch.isfinite(ref)
    assert (got[fin] - ref[fin]).abs().max() <= 2e-5 * max(1.0, ref[fin].abs().max().item())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [[1, 2, 1], [1, 40, 0]])  # (40 tokens of 16 heads: whole tiles in bf16, if `top` is large)
@pytest.mark.parametrize("last,width", [(8129, 0), (9000, 256), (16385, 0), (40000, 0), (9000, 1024), (70400, 0),
                                        (300, 1500)])
@pytest.mark.parametrize("top", [5, 100])
def test_attend_pages_of_long_tables(dtype, new, last, width, top):
    x = Batch([130, last, 64], new, 16, 1, 64, dtype, seed=top, width=width or None)
    c, qs, kl = cache_of(x)
    sc = torch.randn(x.tokens, 1, x.width, generator=torch.Generator().manual_seed(top))
    sc[:, :, 2::5] = 0.5
    sc[1, :, 3::2] = float("nan")
    sc[2, :, :] = float("-inf")
    out, pages = c.attend_pages(x.q.cuda(), sc.cuda(), qs, kl, top=top, sink=1, local=2)
    ref = ref_select(x, sc, top, 1, 2)
    assert torch.equal(pages.cpu(), ref)
    check(out, ref_attend(x, 0.125, pages=ref), dtype)
    capi.pipo_op_paged_check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new", [[1, 1], [20, 1]])
def test_attend_long(dtype, new):
    x = Batch([70001, 8200], new, 16, 1, 64, dtype, seed=3, width=1200)
    c, qs, kl = cache_of(x)
    check(c.attend(x.q.cuda(), qs, kl), ref_attend(x, 0.125), dtype)
    check(c.attend(x.q.cuda(), qs, kl, window=3000), ref_attend(x, 0.125, 3000), dtype)
