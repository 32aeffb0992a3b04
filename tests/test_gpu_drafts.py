"""Verification of drafted tokens on the GPU against whole-number arithmetic, token by token
(tests/paged8_util.py): tokens and counts are equal."""
import pytest
import torch

from paged8_util import verify as ref_verify
from paper_2605_27255_gb300 import capi, drafts

pytestmark = pytest.mark.gpu


def problem(counts, vocab, dtype, seed, sharp=2.0, near=0.7):
    """Target and draft rows, drafts taken from the draft rows, random numbers."""
    g = torch.Generator().manual_seed(seed)
    n, t = len(counts), sum(counts)
    start = torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32)
    logits = torch.randn(t + n, vocab, generator=g) * sharp
    rows = [int(start[b]) + b + i for b in range(n) for i in range(counts[b])]
    draft = torch.softmax(logits[rows] + near * torch.randn(t, vocab, generator=g), -1)
    drafted = (torch.multinomial(draft, 1, generator=g)[:, 0] if t else torch.zeros(0)).to(torch.int32)
    return dict(target=torch.softmax(logits, -1).to(dtype), drafted=drafted, start=start,
                u=torch.rand(t, generator=g), r=torch.rand(n, generator=g)), draft.to(dtype)


def same(x, width, draft=None):
    got = drafts.verify(*(x[k].cuda() for k in ("target", "drafted", "start", "u", "r")), width=width,
                        draft=None if draft is None else draft.cuda())
    want = ref_verify(**x, width=width, draft=draft)
    assert torch.equal(got[1].cpu(), want[1])
    assert torch.equal(got[0].cpu(), want[0])
    return want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 31, 128, 1000, 4096, 5003, 20011])
def test_matches_whole_numbers(dtype, greedy, vocab):
    x, draft = problem([3, 0, 1, 5, 2, 4, 4, 1], vocab, dtype, vocab)
    _, count = same(x, 6, None if greedy else draft)
    if vocab > 100 and not greedy:
        assert count.max() > 1  # some were kept


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_full_vocabulary(dtype):
    x, draft = problem([1, 2], 151936, dtype, 3)
    same(x, 3, draft)
    same(x, 3)


def test_all_kept_none_kept_and_many_drafts():
    """More drafts than a warp looks at in one go; a width that cuts them off."""
    x, draft = problem([70, 40, 33], 300, torch.float32, 5, near=0.0)
    x["u"] *= 0.999
    want = same(x, 71, x["target"][[0 + i for i in range(70)] + [71 + i for i in range(40)] + [112 + i for i in range(33)]])
    assert want[1].tolist() == [71, 41, 34]
    same(x, 71, draft)
    for width in (1, 2, 34, 35, 60):
        same(x, width, draft)
    x["u"][:] = 0.9999999
    same(x, 71, draft)
    x["u"][:] = 0.0
    same(x, 71, draft)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 8), (1, 0), (4, 3), (8, 8)])
def test_strides_and_alignment(dtype, offset, pad):
    """Rows of wider tensors, starting off 16 bytes."""
    vocab = 1003
    x, draft = problem([2, 1, 3], vocab, dtype, 9)
    wide = lambda t: torch.full((t.shape[0], vocab + offset + pad), 9.0, dtype=dtype, device="cuda")  # noqa: E731
    tw, dw = wide(x["target"]), wide(draft)
    tw[:, offset:offset + vocab], dw[:, offset:offset + vocab] = x["target"].cuda(), draft.cuda()
    got = drafts.verify(tw[:, offset:offset + vocab], *(x[k].cuda() for k in ("drafted", "start", "u", "r")), width=4,
                        draft=dw[:, offset:offset + vocab])
    want = ref_verify(**x, width=4, draft=draft)
    assert torch.equal(got[0].cpu(), want[0]) and torch.equal(got[1].cpu(), want[1])


def test_odd_rows():
    """Rows without weight, NaN, negative and infinite values, sums far from one, tokens outside the vocabulary."""
    x, draft = problem([2, 2, 2, 2, 2, 2], 777, torch.float32, 11)
    x["u"][:] = 0.99
    x["target"][0] = 0.0                       # no weight: the draft goes, and the last id is drawn
    x["target"][3] = draft[2] * 0.5            # nothing left of p - q: p itself
    x["target"][6][::3] = float("nan")
    draft[4][::5] = float("nan")
    x["target"][9] *= -1.0
    x["target"][12] = float("inf")
    x["drafted"][10], x["drafted"][8] = -1, 777
    tokens, _ = same(x, 3, draft)
    assert tokens[0, 0] == 776
    same(x, 3)


def test_random_numbers_at_the_edges():
    x, draft = problem([1, 1, 1, 1], 500, torch.float32, 12)
    for r in (0.0, 2.0 ** -24, 0.5, 1 - 2.0 ** -24):
        x["r"][:] = r
        same(x, 2, draft)
    # numbers outside [0, 1) draw the first or the last token with weight
    for r, first in ((-1.0, True), (float("nan"), True), (1.0, False), (7.0, False)):
        x["r"][:] = r
        x["u"][:] = 1.0
        got, _ = drafts.verify(*(x[k].cuda() for k in ("target", "drafted", "start", "u", "r")), width=2)
        x["r"][:] = 0.0 if first else 1 - 2.0 ** -24
        want, _ = ref_verify(**x, width=2)
        assert torch.equal(got.cpu(), want)


def test_tokens_follow_the_targets_distribution():
    """Whatever the drafts were: the first token of 40000 sequences is distributed as the target's row
    (six standard deviations of a count)."""
    n, vocab = 40000, 6
    g = torch.Generator().manual_seed(1)
    p = torch.tensor([0.4, 0.05, 0.25, 0.1, 0.0, 0.2])
    q = torch.tensor([0.1, 0.3, 0.05, 0.25, 0.1, 0.2])
    drafted = torch.multinomial(q, n, replacement=True, generator=g).to(torch.int32)
    tokens, count = drafts.verify(p.cuda().expand(2 * n, vocab).contiguous(), drafted.cuda(),
                                  torch.arange(n + 1, dtype=torch.int32, device="cuda"), torch.rand(n, generator=g).cuda(),
                                  torch.rand(n, generator=g).cuda(), width=2, draft=q.cuda().expand(n, vocab).contiguous())
    have = torch.bincount(tokens[:, 0].cpu().long(), minlength=vocab).double()
    assert have[4] == 0
    assert ((have - n * p.double()).abs() <= 6 * (n * p.double() * (1 - p.double())).sqrt()).all()
    assert abs(count.double().mean().item() - 1 - torch.minimum(p, q).sum().item()) < 6 * 0.5 / n ** 0.5


def test_on_another_stream_and_in_a_graph():
    x, draft = problem([3, 1, 2], 4099, torch.float32, 21)
    dev = {k: v.cuda() for k, v in x.items()}
    d = draft.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        tokens, count = drafts.verify(**dev, width=4, draft=d)
    s.synchronize()
    want = ref_verify(**x, width=4, draft=draft)
    assert torch.equal(tokens.cpu(), want[0]) and torch.equal(count.cpu(), want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tokens, count = drafts.verify(**dev, width=4, draft=d)
    for seed in (5, 6):
        y = torch.Generator().manual_seed(seed)
        x["u"], x["r"] = torch.rand(6, generator=y), torch.rand(3, generator=y)
        x["start"] = torch.tensor([0, 2, 4, 6] if seed == 5 else [0, 0, 3, 6], dtype=torch.int32)
        for k in ("u", "r", "start"):
            dev[k].copy_(x[k])
        g.replay()
        want = ref_verify(**x, width=4, draft=draft)
        assert torch.equal(tokens.cpu(), want[0]) and torch.equal(count.cpu(), want[1])


def test_refusals():
    x, draft = problem([3, 1, 2], 64, torch.float32, 2)
    dev = {k: v.cuda() for k, v in x.items()}
    d = draft.cuda()
    for k, v in (("target", dev["target"][:-1]), ("target", dev["target"].half()), ("target", x["target"]),
                 ("drafted", dev["drafted"].long()), ("start", dev["start"][:-1]), ("u", dev["u"].double()),
                 ("u", dev["u"][:-1]), ("r", dev["r"].bfloat16()), ("start", dev["start"].cpu())):
        with pytest.raises(ValueError):
            drafts.verify(**{**dev, k: v}, width=4, draft=d)
    for bad in (d[:-1], d.bfloat16(), d[:, :63], d.cpu()):
        with pytest.raises(ValueError):
            drafts.verify(**dev, width=4, draft=bad)
    for width in (0, -1, 2 ** 20 + 1):
        with pytest.raises(ValueError):
            drafts.verify(**dev, width=width, draft=d)
    with pytest.raises(ValueError, match="gradient"):
        drafts.verify(**{**dev, "target": dev["target"].requires_grad_()}, width=4)
    big = torch.zeros(1, 2 ** 19 + 1, device="cuda")
    with pytest.raises(capi.PipoError):
        drafts.verify(big, dev["drafted"][:0], torch.zeros(2, dtype=torch.int32, device="cuda"), dev["u"][:0], dev["r"][:1], width=1)
    none = drafts.verify(torch.zeros(0, 64, device="cuda"), dev["drafted"][:0], torch.zeros(1, dtype=torch.int32, device="cuda"),
                         dev["u"][:0], dev["r"][:0], width=3)
    assert none[0].shape == (0, 3) and none[1].shape == (0,)
