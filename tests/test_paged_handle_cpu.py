"""What ``paged.PagedCache`` does on the host, with the library's calls, the
stream and the capture state replaced by stand-ins and CPU tensors in place of
device tensors: nothing is launched."""
import types

import pytest
import torch

from paper_2605_27255_gb300 import capi, paged


class Host:
    """The state that the stand-ins report, and what they were given."""

    def __init__(self):
        self.stream, self.capturing = 0, False
        self.scratch = []    # (address, bytes) of every attention call
        self.allocated = {}  # address of a new tensor -> (stream, capturing) at its allocation
        self.kept = []       # those tensors: an address stays one tensor's


@pytest.fixture
def host(monkeypatch):
    h = Host()
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    monkeypatch.setattr(paged, "_raw_stream", lambda index: h.stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: h.capturing)
    monkeypatch.setattr(capi, "pipo_op_attn_paged_scratch", lambda c, tokens: 1000 * tokens)

    def empty(*args, **kw):
        t = torch.zeros(*args, **kw)
        h.allocated[t.data_ptr()] = (h.stream, h.capturing)
        h.kept.append(t)
        return t

    stand_in = types.SimpleNamespace(**{k: getattr(torch, k) for k in dir(torch) if not k.startswith("__")})
    stand_in.empty = empty
    monkeypatch.setattr(paged, "torch", stand_in)
    monkeypatch.setattr(capi, "pipo_op_attn_paged", lambda *a: h.scratch.append(a[8:10]))
    return h


def cache(batch=2, pages=3, n_q=4, n_kv=2, d_h=64):
    pool = lambda: torch.zeros(batch * pages, n_kv, paged.PAGE, d_h)  # noqa: E731
    return paged.PagedCache(pool(), pool(), torch.zeros(batch, pages, dtype=torch.int32), n_q=n_q)


def attend(c, tokens, **kw):
    q_start = torch.tensor([0] + [tokens] * c.table.shape[0], dtype=torch.int32)
    return c.attend(torch.zeros(tokens, c.n_q, c.d_h), q_start, torch.zeros(c.table.shape[0], dtype=torch.int32), **kw)


def test_a_captured_call_has_scratch_of_the_capture(host):
    """A graph writes its scratch at every replay: memory that was allocated while it was
    captured is the graph's, anything else may be given to another tensor by then (a larger call
    takes a new buffer).  Eager calls in turn stay off a graph's memory."""
    c = cache()
    attend(c, 2)
    host.capturing = True
    attend(c, 2)
    attend(c, 5)
    host.capturing = False
    attend(c, 400)
    attend(c, 2)
    for (address, size), (tokens, captured) in zip(host.scratch, [(2, 0), (2, 1), (5, 1), (400, 0), (2, 0)]):
        assert size >= 1000 * tokens
        assert host.allocated[address] == (0, bool(captured))


def test_scratch_belongs_to_the_stream_that_uses_it(host):
    """The allocator orders the next use of a buffer behind the work of the stream that it was
    allocated on, and no other."""
    c = cache()
    for stream, tokens in [(0, 4), (7, 4), (0, 4), (7, 90), (0, 50), (0, 3)]:
        host.stream = stream
        attend(c, tokens)
        address, size = host.scratch[-1]
        assert size >= 1000 * tokens and host.allocated[address] == (stream, False)
    # the calls of a stream share a buffer while it is large enough
    assert host.scratch[0] == host.scratch[2] and host.scratch[4] == host.scratch[5]
