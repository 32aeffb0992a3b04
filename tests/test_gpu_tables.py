"""Block tables on the GPU against the same steps taken request by request."""
import random

import pytest
import torch

from paged8_util import tables as ref_tables
from paged_util import PAGE
from paper_2605_27255_gb300 import capi, paged

pytestmark = pytest.mark.gpu


class State:
    """The library's tables and the reference's, step by step."""

    def __init__(self, batch, max_pages, n_blocks):
        self.t = paged.BlockTables.new(batch, max_pages, n_blocks)
        self.table = [[-1] * max_pages for _ in range(batch)]
        self.held, self.free, self.n_free = [0] * batch, list(range(n_blocks)), n_blocks

    def step(self, kept, added, tokens):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        got = self.t.advance(i32(kept), i32(added), tokens)
        self.n_free, *ref = ref_tables(self.table, self.held, self.free, self.n_free, kept, added, tokens)
        for name, have, want in zip(("q_start", "kv_len", "slots", "positions"), got, ref):
            assert have.tolist() == want, name
        self.same()
        return ref

    def same(self):
        assert self.t.table.tolist() == self.table
        assert self.t.held.tolist() == self.held
        assert self.t.free.tolist() == self.free
        assert self.t.n_free.tolist() == [self.n_free]
        live = self.free[:self.n_free] + [x for row in self.table for x in row if x >= 0]
        assert sorted(live) == list(range(len(self.free)))  # every block has one holder


@pytest.mark.parametrize("batch,max_pages,n_blocks,longest,seed", [
    (1, 1, 1, 64, 0), (1, 40, 33, 700, 1), (5, 8, 20, 200, 2), (33, 20, 300, 500, 3), (257, 9, 900, 300, 4),
    (1024, 5, 2500, 120, 5), (1025, 5, 2500, 120, 6), (4096, 4, 7000, 90, 7), (64, 60, 1500, 3700, 8)])
def test_steps_match_the_reference(batch, max_pages, n_blocks, longest, seed):
    """Growth, rollback, ends, requests that do not fit: ten steps in a row."""
    rng = random.Random(seed)
    s = State(batch, max_pages, n_blocks)
    lens = [0] * batch
    for _ in range(10):
        kept = [0 if rng.random() < 0.15 else max(0, n - rng.randrange(6)) if rng.random() < 0.5 else n for n in lens]
        added = [rng.randrange(1, longest) if k == 0 else rng.randrange(0, 6) for k in kept]
        room = sum(added) if rng.random() < 0.7 else sum(added) * 2 // 3
        _, lens, _, _ = s.step(kept, added, room)


def test_the_same_call_again_changes_nothing():
    s = State(6, 10, 40)
    s.step([0] * 6, [100, 64, 1, 0, 300, 65], 600)
    first = s.step([90, 10, 1, 0, 300, 65], [30, 200, 64, 5, 0, 1], 400)
    state = [t.clone() for t in (s.t.table, s.t.held, s.t.free, s.t.n_free)]
    again = s.step([90, 10, 1, 0, 300, 65], [30, 200, 64, 5, 0, 1], 400)
    assert first == again
    for a, b in zip(state, (s.t.table, s.t.held, s.t.free, s.t.n_free)):
        assert torch.equal(a, b)


def test_without_blocks_rows_or_tokens():
    s = State(4, 4, 6)
    s.step([0] * 4, [128, 128, 64, 0], 320)         # one block is left
    q, kv, _, _ = s.step([128, 128, 64, 0], [1, 1, 129, 1], 200)
    assert kv == [129, 128, 64, 0]                  # the first takes it, the others wait
    q, kv, _, _ = s.step([129, 128, 64, 0], [0, 200, 0, 0], 200)
    assert kv[1] == 128                             # its row has no room
    q, kv, _, _ = s.step([129, 100, 64, 0], [5, 6, 0, 0], 10)
    assert kv == [134, 100, 64, 0]                  # no rows for the second's tokens
    s.step([0, 0, 0, 0], [0, 0, 0, 0], 0)
    assert s.n_free == 6


def test_odd_numbers():
    """More kept than held, negative numbers, tokens beyond any table: clamped or not served."""
    s = State(3, 5, 9)
    s.step([5, -7, 2 ** 31 - 1], [-3, 2 ** 31 - 1, 10], 40)
    s.step([64 * 5 + 1, 2 ** 31 - 1, 2 ** 31 - 1], [64, 64, 2 ** 31 - 1], 40)


def test_a_state_that_is_not_one_writes_nothing_outside():
    """Counts beyond the tables are clamped (the result is as meaningless as the state, the memory around is
    not touched)."""
    buf = torch.full((4, 64), -9, dtype=torch.int32, device="cuda")
    table, free = buf[1, :12].view(3, 4), buf[2, :7]
    held = torch.tensor([100, -5, 4], dtype=torch.int32, device="cuda")
    n_free = torch.tensor([1000], dtype=torch.int32, device="cuda")
    t = paged.BlockTables(table, held, free, n_free)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    t.advance(i32([0, 3, 70]), i32([500, 64, 3]), 200)
    n_free.fill_(-4)
    t.advance(i32([0, 3, 70]), i32([50, 64, 3]), 200)
    torch.cuda.synchronize()
    assert (buf[0] == -9).all() and (buf[3] == -9).all() and (buf[1, 12:] == -9).all() and (buf[2, 7:] == -9).all()
    assert (held >= 0).all() and (held <= 4).all()


@pytest.mark.parametrize("tokens", [4096, 4097, 70000])
def test_many_tokens(tokens):
    s = State(7, 300, 1300)
    a = tokens // 4
    s.step([0] * 7, [a, 0, 17, 1, a, 0, a], tokens)


def test_in_a_graph_and_in_place():
    """kv_len of one step is the kept lengths of the next; a graph follows the lengths."""
    s = State(3, 8, 20)
    kept = torch.zeros(3, dtype=torch.int32, device="cuda")
    added = torch.tensor([70, 5, 64], dtype=torch.int32, device="cuda")
    out = [torch.empty(4, dtype=torch.int32, device="cuda")] + \
        [torch.empty(200, dtype=torch.int32, device="cuda") for _ in range(2)]

    def call():
        capi.pipo_op_page_tables(s.t._p, kept.data_ptr(), added.data_ptr(), 200, out[0].data_ptr(), kept.data_ptr(),
                                 out[1].data_ptr(), out[2].data_ptr(), torch.cuda.current_stream().cuda_stream)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    lens = [0, 0, 0]
    for add in ([70, 5, 64], [1, 1, 1], [60, 0, 2], [1, 1, 100]):
        added.copy_(torch.tensor(add, dtype=torch.int32))
        g.replay()
        s.n_free, q, lens, slots, pos = ref_tables(s.table, s.held, s.free, s.n_free, lens, add, 200)
        assert out[0].tolist() == q and kept.tolist() == lens and out[1].tolist() == slots and out[2].tolist() == pos
        s.same()


def test_refusals():
    t = paged.BlockTables.new(3, 5, 9)
    z = torch.zeros(3, dtype=torch.int32, device="cuda")
    for kept, added in ((z[:2], z), (z, z.long()), (z, z.cpu()), (torch.zeros(6, dtype=torch.int32, device="cuda")[::2], z)):
        with pytest.raises(ValueError):
            t.advance(kept, added, 4)
    for tokens in (-1, 2 ** 30 + 1):
        with pytest.raises(ValueError):
            t.advance(z, z, tokens)
    with pytest.raises(ValueError):
        paged.BlockTables(t.table, t.held[:2], t.free, t.n_free)
    with pytest.raises(ValueError):
        paged.BlockTables(t.table.long(), t.held, t.free, t.n_free)
    with pytest.raises(capi.PipoError):
        paged.BlockTables.new(4097, 1, 9).advance(*(torch.zeros(4097, dtype=torch.int32, device="cuda"),) * 2, 0)
    assert PAGE == paged.PAGE
