"""Verification of drafted tokens: clusters that reach their exchange at once, and places that 53 bits do not hold."""
import pytest
import torch

from paper_2605_27255_gb300 import drafts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 3, 9, 129])
def test_short_rows_of_many_sequences(dtype, vocab):
    """Slices that are empty or a few tokens long: a block of a cluster passes its sum on as soon as it has started,
    while others of its cluster may not have.  The weight lies on one token of every row, so that a sum that was lost
    or came to another sequence's block shows as another token.  Calls follow one another without a pause."""
    n = 5000
    g = torch.Generator().manual_seed(vocab)
    at = torch.randint(0, vocab, (n,), generator=g)
    target = torch.zeros(n, vocab)
    target[torch.arange(n), at] = 1.0
    none_i, none_f = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    args = (target.to(dtype).cuda(), none_i, torch.zeros(n + 1, dtype=torch.int32, device="cuda"), none_f,
            torch.rand(n, generator=g).cuda())
    got = [drafts.verify(*args, width=1) for _ in range(20)]
    want = at.to(torch.int32)
    for tokens, count in got:
        assert torch.equal(tokens[:, 0].cpu(), want)
        assert (count == 1).all()


@pytest.mark.parametrize("vocab", [3, 40])
def test_short_rows_without_weight(vocab):
    """Rows that are summed up twice (nothing is left of p - q), beside rows that are summed up once."""
    n = 4000
    g = torch.Generator().manual_seed(vocab)
    at = torch.randint(0, vocab, (2 * n,), generator=g)
    target = torch.zeros(2 * n, vocab)  # two rows a sequence: one draft each
    target[torch.arange(2 * n), at] = 0.5
    draft = 2 * target[::2]
    odd = torch.arange(n) % 2 == 1
    draft[odd] = 0.0
    args = [x.cuda() for x in (target, at[::2].to(torch.int32), torch.arange(n + 1, dtype=torch.int32),
                               torch.full((n,), 1.0 - 2.0 ** -24), torch.rand(n, generator=g))]
    # u q < p: false where q is 2 p (not kept, nothing is left), true where q is 0 (kept, the next row is drawn from)
    want = torch.where(odd, at[1::2], at[::2]).to(torch.int32)
    for _ in range(10):
        tokens, count = drafts.verify(*args, width=2, draft=draft.cuda())
        count = count.cpu()
        assert torch.equal(count, torch.where(odd, 2, 1).to(torch.int32))
        assert torch.equal(tokens.cpu()[torch.arange(n), count - 1], want)


def place(r: float, weights) -> int:
    """The first token whose running weight exceeds floor(r W), in whole numbers (r = m / 2^s exactly)."""
    m, d = r.as_integer_ratio()
    goal, total = m * sum(weights) // d, 0
    for v, w in enumerate(weights):
        total += w
        if total > goal:
            return v


@pytest.mark.parametrize("n", [1025, 2049, 65537, 1 << 19])
@pytest.mark.parametrize("r", [0.5, 0.25, 1 - 2.0 ** -24, 0.75 + 2.0 ** -24, 2.0 ** -9, 2.0 ** -30, 2.0 ** -140, 0.0])
def test_places_that_53_bits_do_not_hold(n, r):
    """Rows of ones (they need not add up to one): W = n 2^44 - 1 in units of 2^-44, so that r W ends just below whole
    tokens, and a product rounded to 53 bits on them."""
    row = torch.ones(1, n)
    row[0, n - 2] = 1 - 2.0 ** -24  # 2^20 units less
    row[0, n - 1] = (2 ** 20 - 1) * 2.0 ** -44  # 2^20 - 1 more
    one = 1 << 44
    weights = [one] * (n - 2) + [one - (1 << 20), (1 << 20) - 1]
    assert sum(weights) == (n - 1) * one - 1
    none_i, none_f = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, device="cuda")
    tokens, _ = drafts.verify(row.cuda(), none_i, torch.zeros(2, dtype=torch.int32, device="cuda"), none_f,
                              torch.tensor([r], device="cuda"), width=1)
    assert tokens.item() == place(r, weights)
