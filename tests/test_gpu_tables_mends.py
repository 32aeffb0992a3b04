"""Block tables: sequences that are said to keep more entries than their blocks hold."""
import pytest
import torch

from paged_util import PAGE
from test_gpu_tables import State

pytestmark = pytest.mark.gpu


def test_keeping_more_than_is_held_is_clamped_at_every_call():
    """The same call again: clamped to what the call before has left, so each one takes a block more."""
    s = State(2, 8, 20)
    s.step([0, 0], [64, 64], 128)  # one block each
    for held in (1, 2, 3):
        q_start, kv_len, slots, positions = s.step([1000, 64], [64, 0], 128)
        assert kv_len == [PAGE * (held + 1), 64]
        assert positions[:64] == list(range(PAGE * held, PAGE * (held + 1)))
        assert s.held == [held + 1, 1]


def test_a_sequence_that_is_not_served_reports_what_it_keeps():
    """No room for its tokens: the length is the clamped one, and the blocks stay."""
    s = State(2, 8, 20)
    s.step([0, 0], [70, 64], 256)  # two blocks, one
    q_start, kv_len, _, _ = s.step([1000, 64], [64, 1], 32)
    assert kv_len == [2 * PAGE, 64] and q_start == [0, 0, 0]
    assert s.held == [2, 1]
    # within what is held the same call changes nothing
    state = [t.clone() for t in (s.t.table, s.t.held, s.t.free, s.t.n_free)]
    for _ in range(2):
        s.step([128, 64], [1, 1], 32)
        now = [t.clone() for t in (s.t.table, s.t.held, s.t.free, s.t.n_free)]
        assert now[1].tolist() == [3, 2]
    again = s.step([128, 64], [1, 1], 32)
    assert again[1] == [129, 65]
    for a, b in zip(now, (s.t.table, s.t.held, s.t.free, s.t.n_free)):
        assert torch.equal(a, b)
    assert not torch.equal(state[1], now[1])
