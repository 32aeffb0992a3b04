"""The handles of the 8-bit cache, the block tables and the verification on the host (stand-ins
as in test_paged_handle_cpu.py), what the library refuses before any CUDA call, and the
reference functions of the GPU tests against what they say."""
import ctypes

import pytest
import torch

import paged8_util
from paged_util import PAGE
from paper_2605_27255_gb300 import capi, drafts, paged
from test_capi_cpu import struct_fields
from test_paged_handle_cpu import host  # noqa: F401


def cache8(batch=2, pages=3, n_q=4, n_kv=2, d_h=64):
    pool = lambda: torch.zeros(batch * pages, n_kv, PAGE, d_h, dtype=torch.uint8).view(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.ones(batch * pages, n_kv)  # noqa: E731
    return paged.PagedCache8(pool(), pool(), scale(), scale(), torch.zeros(batch, pages, dtype=torch.int32), n_q=n_q)


@pytest.fixture
def host8(host, monkeypatch):  # noqa: F811
    def stands_in(name, fn):
        def call(*a):
            host.calls.append((name, host.device))
            return fn(*a)
        monkeypatch.setattr(capi, name, call)

    stands_in("pipo_op_attn_paged8_scratch", lambda c, tokens: 1000 * tokens)
    stands_in("pipo_op_attn_paged8", lambda *a: host.scratch.append(a[8:10]))
    stands_in("pipo_op_kv_append8", lambda *a: None)
    stands_in("pipo_op_page_tables", lambda *a: None)
    stands_in("pipo_op_verify_drafts", lambda *a: None)
    monkeypatch.setattr(drafts, "_raw_stream", lambda index: host.stream)
    monkeypatch.setattr(drafts, "_current_device", lambda: host.device)
    return host


def attend(c, tokens):
    n = c.table.shape[0]
    return c.attend(torch.zeros(tokens, c.n_q, c.d_h, dtype=torch.bfloat16),
                    torch.tensor([0] + [tokens] * n, dtype=torch.int32), torch.zeros(n, dtype=torch.int32))


def test_the_8_bit_handle_makes_its_own_calls(host8):
    c = cache8()
    out = attend(c, 3)
    assert out.dtype == torch.bfloat16 and out.shape == (3, 4, 64)
    k = torch.zeros(3, 2, 64)
    qs, kl = torch.tensor([0, 3, 3], dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    assert c.append(torch.zeros(3, 4, 64), k, k, qs, kl).dtype == torch.bfloat16
    assert {n for n, _ in host8.calls} == {"pipo_op_attn_paged8_scratch", "pipo_op_attn_paged8", "pipo_op_kv_append8"}
    assert not hasattr(c, "page_scores") and not hasattr(c, "attend_pages")


def test_scratch_of_the_8_bit_handle(host8):
    """Per stream, and a capture's own from the graph's pool."""
    c = cache8()
    for stream, capturing, tokens in [(0, False, 4), (7, False, 4), (0, True, 4), (0, False, 90), (7, False, 2)]:
        host8.stream, host8.capturing = stream, capturing
        attend(c, tokens)
        address, size = host8.scratch[-1]
        assert size >= 1000 * tokens and host8.allocated[address] == (stream, capturing)
    assert host8.scratch[1] == host8.scratch[4]


def test_calls_run_on_the_tensors_device(host8):
    c = cache8()
    t = paged.BlockTables.new(2, 3, 9, "cpu")
    z = torch.zeros(2, dtype=torch.int32)
    c.index = t.index = 1
    host8.device = 0
    attend(c, 3)
    t.advance(z, z, 5)
    assert host8.device == 0 and host8.calls and all(d == 1 for _, d in host8.calls)


def test_tensors_that_the_handles_refuse(host8):
    c = cache8()
    pool, scale, table = c.k, c.k_scale, c.table
    for bad in [(pool.view(torch.uint8), pool, scale, scale, table), (pool[:, :, :32], pool, scale, scale, table),
                (pool, pool[:1], scale, scale, table), (pool, pool, scale.half(), scale, table),
                (pool, pool, scale, scale[:, :1], table), (pool, pool, scale, scale, table.long()),
                (pool, pool, scale, scale.t().contiguous().t(), table)]:
        with pytest.raises(ValueError):
            paged.PagedCache8(*bad, n_q=4)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, requires_grad=True)
    qs, kl = torch.tensor([0, 2, 2], dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="gradient"):
        c.attend(q, qs, kl)
    with torch.no_grad():
        c.attend(q, qs, kl)
    t = paged.BlockTables.new(2, 3, 9, "cpu")
    z = torch.zeros(2, dtype=torch.int32)
    for kept, added, tokens in [(z[:1], z, 1), (z, z.long(), 1), (z, z, -1), (z, z, 2 ** 30 + 1), (z, z, 2 ** 40)]:
        with pytest.raises(ValueError):
            t.advance(kept, added, tokens)
    with pytest.raises(ValueError):
        paged.BlockTables(t.table, t.held, t.free[::2], t.n_free)
    with pytest.raises(ValueError, match="sequences"):
        paged.BlockTables.new(0, 3, 9, "cpu").advance(z[:0], z[:0], 4)


def test_verify_checks_its_tensors(host8):
    x = dict(target=torch.rand(5, 7), drafted=torch.zeros(3, dtype=torch.int32),
             start=torch.tensor([0, 1, 3], dtype=torch.int32), u=torch.rand(3), r=torch.rand(2))
    tokens, count = drafts.verify(**x, width=3, draft=torch.rand(3, 7))
    assert tokens.shape == (2, 3) and count.shape == (2,)
    for k, v in (("target", torch.rand(4, 7)), ("target", torch.rand(5, 7).double()), ("target", torch.rand(7, 5).t()),
                 ("drafted", x["drafted"].long()), ("start", x["start"][:2]), ("u", torch.rand(2)),
                 ("r", torch.rand(2).double()), ("u", torch.rand(6)[::2]), ("drafted", x["drafted"][None]),
                 ("target", torch.tensor(1.0)), ("r", torch.tensor(0.5)), ("start", torch.tensor(0, dtype=torch.int32))):
        with pytest.raises(ValueError):
            drafts.verify(**{**x, k: v}, width=3)
    for draft in (torch.rand(2, 7), torch.rand(3, 6), torch.rand(3, 7).bfloat16(), torch.rand(3, 7).requires_grad_()):
        with pytest.raises(ValueError):
            drafts.verify(**x, width=3, draft=draft)
    for width in (0, -3, 2 ** 20 + 1, 2 ** 32 + 1):
        with pytest.raises(ValueError):
            drafts.verify(**x, width=width)


A = 1 << 20  # an aligned address that nothing follows


def desc8(**kw):
    c = capi.pipo_paged8(8, 2, 64, 64, 10, 5, 2, A, A, A, A, A, A, A)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def refused(fn, *a):
    with pytest.raises(capi.PipoError) as e:
        fn(*a)
    assert e.value.status == capi.PIPO_EINVAL


def test_what_the_library_refuses_of_an_8_bit_cache():
    row = 8 * 64
    for kw in (dict(head_dim=96), dict(n_kv_heads=3), dict(n_q_heads=34), dict(page_size=32), dict(n_blocks=0),
               dict(max_pages=0), dict(batch=-1), dict(batch=4097), dict(n_blocks=1 << 25)):
        c = desc8(**kw)
        refused(capi.pipo_op_attn_paged8, c, 3, A, row, 0.1, 0, A, row, A, 1 << 30)
        refused(capi.pipo_op_kv_append8, c, 3, 0, A, row, A, 128, A, 128, 0, 0, 1e-6, 0, 0, A)
        assert capi.pipo_op_attn_paged8_scratch(c, 3) == 0
    for kw in (dict(k=0), dict(v=8), dict(k_scale=0), dict(v_scale=2), dict(table=0), dict(q_start=1), dict(kv_len=0)):
        c = desc8(**kw)
        refused(capi.pipo_op_attn_paged8, c, 3, A, row, 0.1, 0, A, row, A, 1 << 30)
        refused(capi.pipo_op_kv_append8, c, 3, 0, A, row, A, 128, A, 128, 0, 0, 1e-6, 0, 0, A)
    c = desc8()
    for a in ((0, row, 0.1, 0, A, row, A), (A, row - 8, 0.1, 0, A, row, A), (A, row + 4, 0.1, 0, A, row, A),
              (A, row, 0.0, 0, A, row, A), (A, row, float("nan"), 0, A, row, A), (A, row, 0.1, -1, A, row, A),
              (A, row, 0.1, 0, A + 8, row, A), (A, row, 0.1, 0, A, row, 0)):
        refused(capi.pipo_op_attn_paged8, c, 3, *a, 1 << 30)
    for a in ((2, A, row, A, 128, A, 128, 0, 0, 1e-6, 0, 0, A), (0, A, row, A, 128, A, 128, 0, 0, -1.0, 0, 0, A),
              (0, A, row, A, 128, A, 128, 0, 0, 1e-6, A, 64, A), (0, A, row, A, 128, A, 128, 0, 0, 1e-6, 0, 0, 0),
              (0, A, row, A, 64, A, 128, 0, 0, 1e-6, 0, 0, A), (0, A, row, A, 128, A, 128, 8, 0, 1e-6, 0, 0, A)):
        refused(capi.pipo_op_kv_append8, c, 3, *a)
    with pytest.raises(capi.PipoError):
        capi._check(capi.load().pipo_op_attn_paged8(None, 3, A, row, 0.1, 0, A, row, A, 1 << 30, None), None)
    # nothing to do: no call into CUDA
    capi.pipo_op_attn_paged8(c, 0, 0, 0, 0.1, 0, 0, 0, 0, 0)
    capi.pipo_op_kv_append8(desc8(batch=0), 5, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1e-6, 0, 0, 0)


def test_what_the_library_refuses_of_tables():
    def tables(**kw):
        p = capi.pipo_page_tables(10, 5, 2, A, A, A, A)
        for k, v in kw.items():
            setattr(p, k, v)
        return p
    for kw in (dict(batch=-1), dict(batch=4097), dict(max_pages=0), dict(max_pages=65535 * 64 + 1), dict(n_blocks=0),
               dict(n_blocks=1 << 25), dict(table=0), dict(held=2), dict(free_blocks=0), dict(n_free=0)):
        refused(capi.pipo_op_page_tables, tables(**kw), A, A, 4, A, A, A, A)
    for a in ((0, A, 4, A, A, A, A), (A, 0, 4, A, A, A, A), (A, A, -1, A, A, A, A), (A, A, (1 << 30) + 1, A, A, A, A),
              (A, A, 4, 0, A, A, A), (A, A, 4, A, 0, A, A), (A, A, 4, A, A, 0, A), (A, A, 4, A, A, A, 2)):
        refused(capi.pipo_op_page_tables, tables(), *a)
    capi.pipo_op_page_tables(tables(batch=0), 0, 0, 0, 0, 0, 0, 0)
    with pytest.raises(capi.PipoError):
        capi._check(capi.load().pipo_op_page_tables(None, A, A, 4, A, A, A, A, None), None)


def test_what_the_library_refuses_of_a_verification():
    good = dict(dtype=0, vocab=7, batch=2, n_drafted=3, target=A, ld_target=7, draft=A, ld_draft=7, drafted=A, start=A,
                u=A, r=A, width=3, tokens=A, count=A)
    for kw in (dict(dtype=2), dict(vocab=0), dict(vocab=2 ** 19 + 1), dict(batch=-1), dict(batch=65537),
               dict(n_drafted=-1), dict(n_drafted=2 ** 30 + 1), dict(width=0), dict(width=2 ** 20 + 1), dict(target=0),
               dict(target=2), dict(ld_target=6), dict(ld_target=2 ** 40 + 1), dict(draft=2), dict(ld_draft=6),
               dict(drafted=0), dict(start=0), dict(u=0), dict(r=2), dict(tokens=0), dict(count=0)):
        refused(capi.pipo_op_verify_drafts, *{**good, **kw}.values())
    capi.pipo_op_verify_drafts(*{**good, "batch": 0, "n_drafted": 0, "target": 0}.values())


def test_structures_match_the_header():
    """Names in the header's order, sizes as a C compiler lays them out (pointers after the 32-bit fields)."""
    for c in (capi.pipo_paged8, capi.pipo_page_tables):
        assert [f for f, _ in c._fields_] == struct_fields(c.__name__)
    assert ctypes.sizeof(capi.pipo_paged8) == 32 + 7 * 8 and capi.pipo_paged8.k.offset == 32
    assert ctypes.sizeof(capi.pipo_page_tables) == 16 + 4 * 8 and capi.pipo_page_tables.table.offset == 16


# ---- what the GPU tests compare with

def test_scales_and_codes():
    for m in (1.0, 0.999, 63.9, 64.0, 1e-3, 5e4):
        s = paged8_util.scale_of(m)
        assert 32 <= m / s < 64 or s == 2.0 ** 7
    assert paged8_util.scale_of(0.0) == 2.0 ** -100 and paged8_util.scale_of(1e30) == 2.0 ** 7
    x = torch.randn(3, 2, PAGE, 64) * torch.tensor([1e-3, 1.0, 0.0])[:, None, None, None]
    codes, scale = paged.encode(x)
    want = torch.full(x.shape, float("nan"), dtype=torch.float64)
    ws = torch.ones(3, 2, dtype=torch.float64)
    paged8_util.put(want, ws, [0, 1, 2], 0, x.transpose(1, 2).reshape(192, 2, 64).double())
    assert torch.equal(codes.double(), want) and torch.equal(scale.double(), ws)
    assert (codes.double() * scale[..., None, None] - x).abs().max() <= 2.0 ** -4 * x.abs().max()


def test_reference_verification_by_hand():
    """A row at a time: kept, refused, drawn."""
    target = torch.tensor([[0.5, 0.25, 0.25], [0.0, 1.0, 0.0], [0.25, 0.25, 0.5], [0.2, 0.2, 0.6]])
    draft = torch.tensor([[0.25, 0.5, 0.25], [0.5, 0.5, 0.0]])
    x = dict(target=target, drafted=torch.tensor([0, 0]), start=torch.tensor([0, 2, 2]), r=torch.tensor([0.0, 0.3]))
    got, count = paged8_util.verify(**x, u=torch.tensor([0.9, 0.0]), width=3, draft=draft)
    # the first draft is twice as likely for the target: kept; the second has probability zero: the rest is token 1
    assert got.tolist() == [[0, 1, -1], [1, -1, -1]] and count.tolist() == [2, 1]
    got, count = paged8_util.verify(**x, u=torch.tensor([0.4, 0.0]), width=2)
    assert got.tolist() == [[0, 1], [1, -1]] and count.tolist() == [2, 1]
    got, _ = paged8_util.verify(**x, u=torch.tensor([0.6, 0.0]), width=3)
    assert got.tolist()[0] == [1, -1, -1]
