"""What ``paged.PagedCache`` does on the host, with the library's calls, the
stream and the capture state replaced by stand-ins and CPU tensors in place of
device tensors: nothing is launched."""
import ctypes
import threading
import types

import pytest
import torch

from paper_2605_27255_gb300 import capi, paged


class Host:
    """The state that the stand-ins report, and what they were given."""

    def __init__(self):
        self.stream, self.capturing = 0, False
        self.device = None   # the thread's current device (that of CPU tensors)
        self.calls = []      # (library call, current device)
        self.scratch = []    # (address, bytes) of every attention call
        self.allocated = {}  # address of a new tensor -> (stream, capturing) at its allocation
        self.kept = []       # those tensors: an address stays one tensor's


@pytest.fixture
def host(monkeypatch):
    h = Host()
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    monkeypatch.setattr(paged, "_raw_stream", lambda index: h.stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: h.capturing)
    monkeypatch.setattr(paged, "_current_device", lambda: h.device, raising=False)

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.outer, h.device = h.device, self.index

        def __exit__(self, *a):
            h.device = self.outer

    monkeypatch.setattr(torch.cuda, "device", Device)

    def stands_in(name, fn):
        def call(*a):
            h.calls.append((name, h.device))
            return fn(*a)
        monkeypatch.setattr(capi, name, call)

    stands_in("pipo_op_attn_paged_scratch", lambda c, tokens: 1000 * tokens)
    stands_in("pipo_op_attn_paged", lambda *a: h.scratch.append(a[8:10]))
    stands_in("pipo_op_attn_pages", lambda *a: h.scratch.append(a[12:14]))
    stands_in("pipo_op_kv_append", lambda *a: None)
    stands_in("pipo_op_page_scores", lambda *a: None)

    def empty(*args, **kw):
        t = torch.zeros(*args, **kw)
        h.allocated[t.data_ptr()] = (h.stream, h.capturing)
        h.kept.append(t)
        return t

    stand_in = types.SimpleNamespace(**{k: getattr(torch, k) for k in dir(torch) if not k.startswith("__")})
    stand_in.empty = empty
    monkeypatch.setattr(paged, "torch", stand_in)
    return h


def cache(batch=2, pages=3, n_q=4, n_kv=2, d_h=64):
    pool = lambda: torch.zeros(batch * pages, n_kv, paged.PAGE, d_h)  # noqa: E731
    return paged.PagedCache(pool(), pool(), torch.zeros(batch, pages, dtype=torch.int32), n_q=n_q,
                            means=torch.zeros(batch * pages, n_kv, d_h))


def batch_of(c, tokens):
    """Queries, q_start and kv_len."""
    n = c.table.shape[0]
    return (torch.zeros(tokens, c.n_q, c.d_h), torch.tensor([0] + [tokens] * n, dtype=torch.int32),
            torch.zeros(n, dtype=torch.int32))


def attend(c, tokens, **kw):
    return c.attend(*batch_of(c, tokens), **kw)


def append(c, tokens, **kw):
    q, qs, kl = batch_of(c, tokens)
    k = torch.zeros(tokens, c.n_kv, c.d_h)
    return c.append(q, k, k, qs, kl, **kw)


def page_scores(c, tokens, **kw):
    return c.page_scores(*batch_of(c, tokens), **kw)


def attend_pages(c, tokens, top=2, **kw):
    q, qs, kl = batch_of(c, tokens)
    return c.attend_pages(q, torch.zeros(tokens, c.n_kv, c.table.shape[1]), qs, kl, top=top, **kw)


CALLS = [append, attend, page_scores, attend_pages]


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


@pytest.mark.parametrize("call", CALLS)
def test_calls_run_on_the_pools_device(host, call):
    """The library launches on the thread's current device, whichever that is; pools on
    another one make it theirs for the call."""
    c = cache()
    c.index = 1
    host.device = 0
    call(c, 3)
    assert host.device == 0
    assert host.calls and all(device == 1 for _, device in host.calls), host.calls
    host.calls.clear()
    host.device = 1
    call(c, 5)
    assert host.calls and all(device == 1 for _, device in host.calls)


def test_threads_do_not_see_each_others_batch(host, monkeypatch):
    """The library reads the batch's pointers after the interpreter lock is let go: a call of
    another thread in between must not change them."""
    c = cache()
    inside, go_on, seen = threading.Event(), threading.Event(), {}

    def kv_append(desc, tokens, *rest):
        if tokens == 3:
            inside.set()
            go_on.wait(5)
        seen[tokens] = (desc.q_start, desc.kv_len)

    monkeypatch.setattr(capi, "pipo_op_kv_append", kv_append)
    batches = {n: batch_of(c, n) for n in (3, 8)}

    def run(n):
        q, qs, kl = batches[n]
        k = torch.zeros(n, c.n_kv, c.d_h)
        c.append(None, k, k, qs, kl)

    first, second = (threading.Thread(target=run, args=(n,)) for n in (3, 8))
    first.start()
    assert inside.wait(5)
    second.start()
    second.join(0.3)  # (it either ends here or waits for the first)
    go_on.set()
    first.join(5)
    second.join(5)
    assert seen == {n: (b[1].data_ptr(), b[2].data_ptr()) for n, b in batches.items()}


def test_integers_past_32_bits_are_not_wrapped(host, monkeypatch):
    """ctypes keeps the low 32 bits of an integer: what the library is given has to be in
    range already, a larger window as the largest there is, other values as ones it refuses."""
    given = []
    monkeypatch.setattr(capi, "pipo_op_attn_paged", lambda *a: given.append([a[5]]))
    monkeypatch.setattr(capi, "pipo_op_attn_pages", lambda *a: given.append(list(a[6:9])))
    c = cache()

    def passed(call, **kw):
        call(c, 2, **kw)
        values = given.pop()
        assert [ctypes.c_int32(v).value for v in values] == values, values
        return values

    for w in (0, 1, 100, 2 ** 31 - 1):
        assert passed(attend, window=w) == [w]
    for w in (2 ** 31, 2 ** 32, 2 ** 32 + 5, 1 << 60):
        assert passed(attend, window=w) == [2 ** 31 - 1]
    for w in (-1, -2 ** 32, -2 ** 32 + 5):
        assert passed(attend, window=w)[0] < 0
    assert passed(attend_pages, top=5, sink=2, local=3) == [5, 2, 3]
    for n in (2 ** 31, 2 ** 32, 2 ** 32 + 1):
        assert passed(attend_pages, sink=n)[1] > 4096 and passed(attend_pages, local=n)[2] > 4096
    for n in (-1, -2 ** 32, -2 ** 32 + 1):
        assert passed(attend_pages, sink=n)[1] < 0 and passed(attend_pages, local=n)[2] < 0
    pool = torch.zeros(2, 2, paged.PAGE, 64)
    wide = paged.PagedCache(pool, pool, torch.zeros(1, 1, dtype=torch.int32), n_q=2 ** 32 + 4)
    assert wide._c.n_q_heads > 65536  # (refused by every call)


def test_inputs_that_require_grad_are_refused(host):
    """The operators have no backward pass: with gradients enabled an output would silently
    carry none."""
    c = cache()

    def inputs():
        q, qs, kl = batch_of(c, 2)
        k, gain = torch.zeros(2, c.n_kv, c.d_h), torch.ones(c.d_h)
        scores = torch.zeros(2, c.n_kv, c.table.shape[1])
        rope = paged.rope_table(c.table.shape[1] * paged.PAGE, c.d_h, 1e4, "cpu")
        return dict(q=q, k=k, v=k.clone(), q_gain=gain, k_gain=gain.clone(), scores=scores, rope=rope), qs, kl

    calls = {
        "q": [lambda x, *b: c.append(x["q"], x["k"], x["v"], *b), lambda x, *b: c.attend(x["q"], *b),
              lambda x, *b: c.page_scores(x["q"], *b), lambda x, *b: c.attend_pages(x["q"], x["scores"], *b, top=1)],
        "k": [lambda x, *b: c.append(None, x["k"], x["v"], *b)],
        "v": [lambda x, *b: c.append(None, x["k"], x["v"], *b)],
        "q_gain": [lambda x, *b: c.append(x["q"], x["k"], x["v"], *b, q_gain=x["q_gain"])],
        "k_gain": [lambda x, *b: c.append(x["q"], x["k"], x["v"], *b, k_gain=x["k_gain"])],
        "rope": [lambda x, *b: c.append(None, x["k"], x["v"], *b, rope=x["rope"])],
        "scores": [lambda x, *b: c.attend_pages(x["q"], x["scores"], *b, top=1)],
    }
    for name, fns in calls.items():
        for fn in fns:
            x, qs, kl = inputs()
            fn(x, qs, kl)
            x[name].requires_grad_()
            with pytest.raises(ValueError, match="gradient"):
                fn(x, qs, kl)
            with torch.no_grad():
                fn(x, qs, kl)
            fn({n: t.detach() for n, t in x.items()}, qs, kl)
