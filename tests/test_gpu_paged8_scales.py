"""Attention over 8-bit pools whose blocks differ in scale by far: what a row does not see, or gives no weight, leaves it
alone.  Errors are measured row by row and dim by dim, against what the row itself attends to.

Tolerance of an output, with weights w_j (64 bits) over the n entries that the row sees, A = sum w_j |v_j| of its dim
and W the largest w_j s_j (s_j the scale of entry j's block):
  2^-8 |out|   the output's rounding, half a bf16 step;
  2^-11 A      a weight's rounding to fp16;
  2^-11 A      its error in fp32, above and below the fraction line: scores below 2^7 in sum over |q k| with some
               sixteen roundings of 2^-24 each come to 2^-13, differences and powers of two to less;
  n 2^-23 W    weights below 2^-14 have a step of 2^-24, half of it lost; they are held times at least 2^7 relative to
               W, and a code is below 2^9."""
import pytest
import torch

from paged8_util import Batch8
from paged_util import PAGE
from paper_2605_27255_gb300 import capi, paged

pytestmark = pytest.mark.gpu

# new tokens with four query heads a kv head: 8, 32 (tiles of few rows), 80 (single tiles), 240 rows (pairs)
TOKENS = [2, 8, 20, 60]


def run(x: Batch8, window=0, scale=None):
    c = paged.PagedCache8(x.k8.cuda(), x.v8.cuda(), x.k_scale.cuda(), x.v_scale.cuda(), x.table.cuda(), n_q=x.x.n_q)
    scale = scale or x.x.d_h ** -0.5
    got = c.attend(x.q.cuda(), x.q_start.cuda(), x.kv_len.cuda(), window=window, scale=scale).cpu().double()
    capi.pipo_op_paged_check()
    assert torch.isfinite(got).all()
    b8, grp = x.x, x.x.n_q // x.x.n_kv
    for t, b, pos in b8.each_token():
        for g in range(b8.n_kv):
            j = torch.arange(max(0, pos - window + 1) if window else 0, pos + 1)
            k, v = b8.rows(x.plain.k, b, g, j), b8.rows(x.plain.v, b, g, j)
            s = x.v_scale.double()[x.table[b].long()[j // PAGE], g]
            q = x.q[t, g * grp:(g + 1) * grp].double()
            assert (scale * q.abs() @ k.abs().T).max() <= 128
            w = torch.softmax(scale * q @ k.T, -1)
            out, A, W = w @ v, w @ v.abs(), (w * s).amax(1, keepdim=True)
            off = (got[t, g * grp:(g + 1) * grp] - out).abs()
            most = 2.0 ** -8 * out.abs() + 2.0 ** -10 * A + len(j) * 2.0 ** -23 * W
            assert (off <= most).all(), (t, g, (off / most).max().item())


def lift(x: Batch8, exps):
    """Page p of every sequence: values times 2^exps(b, p)."""
    for b, n in enumerate(x.x.lens):
        for p in range(-(-n // PAGE)):
            blk, f = x.table[b, p].item(), 2.0 ** exps(b, p)
            x.v_scale[blk] *= f
            x.plain.v[blk] *= f
    return x


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("e", [14, 24, 40, 90])
@pytest.mark.parametrize("far", [-1, 1])
def test_pages_that_the_window_has_passed(d_h, n, e, far):
    """The first tokens' window reaches pages 2^e above (or below) what the last ones see."""
    x = Batch8([300, 299], [n, n], 8, 2, d_h, seed=51)
    lift(x, lambda b, p: far * (e // 2 if p < 3 else e // 2 - e))
    run(x, window=301 - n // 2 - 192)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("e", [14, 24, 40, 90])
def test_pages_of_later_tokens(d_h, n, e):
    """The last tokens begin a page 2^e above the others, which the first ones do not see."""
    x = Batch8([256 + n // 2, 320 + n // 2], [n, n], 8, 2, d_h, seed=52)
    run(lift(x, lambda b, p: e // 2 if p == (4, 5)[b] else e // 2 - e))


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("nats,e", [(10, 8), (10, 16), (10, 40), (10, 120), (10, 185), (30, 40), (30, 48), (30, 130), (60, 80), (60, 100), (60, 185)])
@pytest.mark.parametrize("heavy_first", [True, False])
def test_pages_of_little_weight(d_h, n, nats, e, heavy_first):
    """Pages of scores `nats` below the others, with values 2^e above them: the one, the other, or both make the sum,
    and the weights' sum is that of the pages of small values."""
    x = Batch8([400, 330], [n, n], 8, 2, d_h, seed=53)
    heavy = lambda p: (p < 3) == heavy_first  # noqa: E731
    x.q[..., 0] = 32.0
    half = nats / 2 * d_h ** 0.5 / 32  # of dim 0
    for b, length in enumerate(x.x.lens):
        for p in range(-(-length // PAGE)):
            blk = x.table[b, p].item()
            code = (half / x.k_scale[blk] * (1 if heavy(p) else -1)).to(torch.float8_e4m3fn)
            x.k8[blk, :, :, 0] = code[:, None].expand(2, PAGE)
            x.plain.k[blk, :, :, 0] = (code.double() * x.k_scale[blk].double())[:, None]
    run(lift(x, lambda b, p: e // 2 - e if heavy(p) else e // 2))


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("new", [[2, 1], [8, 5], [20, 18], [60, 90]])
@pytest.mark.parametrize("window", [0, 500])
@pytest.mark.parametrize("odd", [False, True])
def test_every_page_its_own_scale(d_h, new, window, odd):
    """Scales from 2^-45 to 2^45 in any order, over items that several workers share; odd: no powers of two."""
    g = torch.Generator().manual_seed(54)
    x = Batch8([2500, 900], new, 8, 2, d_h, seed=54)
    e = torch.randint(-45, 46, (2, 40), generator=g).double()
    if odd:
        e += torch.rand(2, 40, generator=g).double()
        x.v_scale, x.plain.v = x.v_scale.double(), x.plain.v
        lift(x, lambda b, p: e[b, p].item())
        x.v_scale = x.v_scale.float()
        x.plain.v = x.v8.double() * x.v_scale[..., None, None].double()
    else:
        lift(x, lambda b, p: e[b, p].item())
    run(x, window)


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("size", [1e4, 1e6, 1e12])
def test_large_scores_keep_the_scales(d_h, n, size):
    """Scores so large that one entry has all the weight: its value comes out, whatever the scales of the others are."""
    x = lift(Batch8([300, 299], [n, n], 8, 2, d_h, seed=55), lambda b, p: (-7.3, 9, 0.4, -20, 3.6)[p])
    x.v_scale = x.v_scale.float()
    x.plain.v = x.v8.double() * x.v_scale[..., None, None].double()
    c = paged.PagedCache8(x.k8.cuda(), x.v8.cuda(), x.k_scale.cuda(), x.v_scale.cuda(), x.table.cuda(), n_q=8)
    got = c.attend(x.q.cuda(), x.q_start.cuda(), x.kv_len.cuda(), scale=size).cpu().double()
    seen = 0
    for t, b, pos in x.x.each_token():
        for h in range(8):
            j = torch.arange(pos + 1)
            k, v = x.x.rows(x.plain.k, b, h // 4, j), x.x.rows(x.plain.v, b, h // 4, j)
            s = x.q[t, h].double() @ k.T
            top = s.topk(2)[0]
            # (fp32 scores are off by 2^-20 of sum |q k| at most: 60 nats apart leave less weight than 2^-86 to each of
            # the others, on values below 2^12)
            if (top[0] - top[1]) * size < 60 + 2.0 ** -19 * size * (x.q[t, h].double().abs() @ k.abs().T).max():
                continue
            seen += 1
            want = v[s.argmax()]
            assert ((got[t, h] - want).abs() <= (2.0 ** -8 + 2.0 ** -10) * want.abs() + 2.0 ** -65).all()
    assert seen > 0.9 * 16 * n


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("n", TOKENS)
@pytest.mark.parametrize("small_first", [True, False])
def test_parts_whose_scales_lie_at_the_ends(d_h, n, small_first):
    """Items that many workers share, half of their entries with values near 2^-96 and half near 2^91: all weights
    count below the fraction line, whichever part they come from."""
    x = Batch8([4500, 3800], [n, n], 8, 2, d_h, seed=56)
    run(lift(x, lambda b, p: -95 if (p < 34) == small_first else 94))
