"""Attention over 8-bit pools: queries whose dims differ in size by far keep their digits, however many rows share a tile.

Tolerance of an output, with weights w_j (64 bits) over the n entries that the row sees, A = sum w_j |v_j| of its dim and
W the largest w_j s_j (s_j the scale of entry j's block): 2^-8 |out| + 2^-10 A + n 2^-23 W as for rows of one size
(output, weights in fp16, scores in fp32), and what the queries lose: dims from 2^-23 of the row's largest on are exact,
each below is off by 2^-31 of the largest at most; a score is then off by d_j = scale sum |loss| |k_j|, every weight by a
factor within exp(+-2 max d), above and below the fraction line."""
import pytest
import torch

from paged8_util import Batch8
from paper_2605_27255_gb300 import capi, paged

pytestmark = pytest.mark.gpu

# new tokens with four query heads a kv head: 8, 32 (tiles of few rows), 80 (single tiles), 240 rows (pairs)
TOKENS = [2, 8, 20, 60]


def run(x: Batch8):
    c = paged.PagedCache8(x.k8.cuda(), x.v8.cuda(), x.k_scale.cuda(), x.v_scale.cuda(), x.table.cuda(), n_q=x.x.n_q)
    scale = x.x.d_h ** -0.5
    got = c.attend(x.q.cuda(), x.q_start.cuda(), x.kv_len.cuda(), scale=scale).cpu().double()
    capi.pipo_op_paged_check()
    grp = x.x.n_q // x.x.n_kv
    for t, b, pos in x.x.each_token():
        for g in range(x.x.n_kv):
            j = torch.arange(pos + 1)
            k, v = x.x.rows(x.plain.k, b, g, j), x.x.rows(x.plain.v, b, g, j)
            s = x.v_scale.double()[x.table[b].long()[j // 64], g]
            q = x.q[t, g * grp:(g + 1) * grp].double()
            assert (scale * q.abs() @ k.abs().T).max() <= 128
            most = q.abs().amax(1, keepdim=True)
            loss = torch.where(q.abs() < 2.0 ** -23 * most, 2.0 ** -31 * most, 0.0)
            grow = torch.expm1(2 * scale * (loss @ k.abs().T).amax(1, keepdim=True))
            w = torch.softmax(scale * q @ k.T, -1)
            out, A, W = w @ v, w @ v.abs(), (w * s).amax(1, keepdim=True)
            off = (got[t, g * grp:(g + 1) * grp] - out).abs()
            assert (off <= 2.0 ** -8 * out.abs() + (2.0 ** -10 + 2 * grow) * A + len(j) * 2.0 ** -23 * W).all(), (t, g)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("exp", [8, 10, 12, 14, 16, 20])
def test_one_dim_far_above_the_others(d_h, n, exp):
    """A dim 2^exp times the rest of its row, which the keys do not have: the scores are those of the rest."""
    x = Batch8([400, 330], [n, n], 8, 2, d_h, seed=61)
    x.q[..., 3] = (x.q[..., 3].float().sign() * 2.0 ** exp).bfloat16()
    x.k8[..., 3] = 0.0
    x.plain.k[..., 3] = 0.0
    run(x)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("size", [2.0 ** -60, 1.0, 2.0 ** 60])
def test_dims_of_every_size(d_h, n, size):
    """Queries from 1 down to 2^-12 of a row's largest, on keys that make up for it: every dim counts as much as any
    other.  Rows of very small and very large queries, on keys that make up for that too."""
    x = Batch8([400, 330], [n, n], 8, 2, d_h, seed=62)
    g = torch.Generator().manual_seed(63)
    r = torch.randint(0, 13, (d_h,), generator=g).double()
    r[:2] = torch.tensor([0.0, 12.0])
    x.q = (x.q.double() * 2.0 ** -r * size).bfloat16()
    x.plain.q = x.q
    x.k8 = (torch.randn(x.k8.shape, generator=g) * (2.0 ** (r - 6)).float()).to(torch.float8_e4m3fn)
    x.k_scale = torch.full_like(x.k_scale, 2.0 ** 6 / size)
    x.plain.k = x.k8.double() * x.k_scale[..., None, None].double()
    run(x)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
def test_rows_of_the_smallest_numbers(d_h, n):
    """Queries at the low end of bf16, its subnormals among them, on keys of 2^100 and more: scores of about one."""
    x = Batch8([400, 330], [n, n], 8, 2, d_h, seed=64)
    x.q = (x.q.double() * 2.0 ** -110).bfloat16()
    x.q[:, ::2] = (x.q[:, ::2].double() * 2.0 ** -16).bfloat16()  # 2^-126 and below
    x.plain.q = x.q
    x.k_scale = torch.full_like(x.k_scale, 2.0 ** 100)
    x.plain.k = x.k8.double() * 2.0 ** 100
    x.q[:, 1::2] = (x.q[:, 1::2].double() * 2.0 ** 4).bfloat16()
    run(x)
