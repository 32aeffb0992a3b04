"""Append to blocks that something else has filled: scales above 2^7 and between powers of two.

A stored value is within half a step of the entry: 2^-4 of its magnitude, or 2^-10 of the scale where it is
subnormal; the division by a scale that is no power of two is a product with a rounded reciprocal, two fp32 roundings
(2^-22 holds them)."""
import math

import pytest
import torch

from paged8_util import TOP, scale_of
from paged_util import PAGE
from paper_2605_27255_gb300 import paged

pytestmark = pytest.mark.gpu


def filled(scale, held, d_h=64, seed=0):
    """One block with `held` entries of random codes (all digits, both signs) under `scale`."""
    g = torch.Generator().manual_seed(seed)
    raw = torch.randint(0, 256, (1, 2, PAGE, d_h), generator=g, dtype=torch.uint8)
    raw[(raw & 0x7f) == 0x7f] = 0x7e
    codes = raw.cuda().view(torch.float8_e4m3fn)
    s = torch.full((1, 2), scale, device="cuda")
    return paged.PagedCache8(codes, codes.clone(), s, s.clone(), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), n_q=2)


def add(c, x, held):
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    c.append(None, x.cuda(), (-x).cuda(), i32(0, x.shape[0]), i32(held + x.shape[0]))


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("held,n", [(1, 1), (63, 1), (5, 40)])
@pytest.mark.parametrize("scale", [128.0, 200.0, 1024.0, 3e5, 2.0 ** 100])
@pytest.mark.parametrize("over", [0.5, 1.5, 50.0])
def test_a_scale_above_the_chosen_ones_stays(scale, over, held, n, d_h):
    """Entries that do not fit saturate; what the block holds keeps its codes and its scale."""
    c = filled(scale, held, d_h)
    before = c.k.view(torch.uint8).clone()
    x = torch.full((n, 2, d_h), TOP * scale * over)
    x[:, :, 1::2] = scale
    add(c, x, held)
    assert (c.k_scale == scale).all() and (c.v_scale == scale).all()
    for pool, sign in ((c.k, 1), (c.v, -1)):
        assert torch.equal(pool.view(torch.uint8)[:, :, :held], before[:, :, :held])
        assert torch.equal(pool.view(torch.uint8)[:, :, held + n:], before[:, :, held + n:])
        got = pool[0, :, held:held + n].float()
        assert (got[..., 0::2] == sign * TOP * min(over, 1.0)).all() and (got[..., 1::2] == sign).all()


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-6, 0.3, 1.0, 5.7, 127.0])
@pytest.mark.parametrize("size", [1.0, 40.0, 700.0, 3e4, 1e6])
def test_any_scale_below_grows_as_its_own_do(scale, size, d_h):
    """A scale that is no power of two is left for one when an entry does not fit: held values are rounded once more,
    none of them saturates, and the new ones are as near as under their own scale."""
    held, n = 20, 3
    c = filled(scale, held, d_h, seed=3)
    old = c.k_scale.cpu()[0, 0].item()
    before = c.k[0, :, :held].double().cpu() * old
    x = torch.randn(n, 2, d_h, generator=torch.Generator().manual_seed(4)) * size
    add(c, x, held)
    for pool, scales, sign in ((c.k, c.k_scale, 1), (c.v, c.v_scale, -1)):
        for g in range(2):
            most = x[:, g].abs().max().item()
            now = scales[0, g].item()
            # (450: entries within a fp32 rounding of 448 times the scale go either way; none of these is)
            assert not TOP * old <= most < 450 * old
            assert now == (max(scale_of(most), old) if most > TOP * old else old)
            held_now, held_was = pool[0, g, :held].double().cpu() * now, before[g]
            off = (held_now - held_was).abs()
            if now == old:
                assert (off == 0).all()
            else:
                assert (off <= torch.maximum(2.0 ** -4 * held_was.abs(), torch.tensor(2.0 ** -10 * now)) * (1 + 2.0 ** -20)).all()
            new_now, want = pool[0, g, held:held + n].double().cpu() * now, sign * x[:, g].double().clamp(-TOP * now, TOP * now)
            off = (new_now - want).abs()
            assert (off <= torch.maximum(2.0 ** -4 * want.abs(), torch.tensor(2.0 ** -10 * now)) * (1 + 2.0 ** -20)).all()
            assert math.isfinite(now) and now >= old


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("large", [100.0, 3000.0, 5e4])
def test_a_draft_that_is_given_up_leaves_its_scale(d_h, large):
    """Entries kept before a large draft, and those appended in its place: the scale stays as high as the draft needed,
    every entry is within its half step and a subnormal step of it (half of one each time it is rounded, and scales at
    least double)."""
    pool = lambda: torch.zeros(1, 2, PAGE, d_h, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
    s = lambda: torch.ones(1, 2, device="cuda")  # noqa: E731
    c = paged.PagedCache8(pool(), pool(), s(), s(), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), n_q=2)
    g = torch.Generator().manual_seed(9)
    x = torch.randn(12, 2, d_h, generator=g)
    add(c, x[:8], 0)
    first = c.k_scale.clone()
    add(c, torch.full((2, 2, d_h), large), 8)  # two drafts, given up
    raised = c.k_scale.clone()
    assert (raised == scale_of(large)).all() and (raised > first).all()
    add(c, x[8:], 8)
    for pool, scales, sign in ((c.k, c.k_scale, 1), (c.v, c.v_scale, -1)):
        assert torch.equal(scales, raised)
        got = pool[0, :, :12].double().cpu().transpose(0, 1) * scale_of(large)
        want = sign * x.double()
        assert ((got - want).abs() <= 2.0 ** -4 * want.abs() * (1 + 2.0 ** -4) + 2.0 ** -9 * scale_of(large)).all()
