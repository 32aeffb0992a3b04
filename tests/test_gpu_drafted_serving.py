"""The operators of a drafting server in a row, as examples/drafted_layer.py uses them: tables, append to the
8-bit cache, attention over it, verification."""
import importlib.util
import os
import random

import pytest
import torch

from paper_2605_27255_gb300 import capi, drafts, paged

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_layer.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("drafted_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def prompts_of(vocab, lens, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, vocab, (n,), generator=g).tolist() for n in lens]


def check_greedy(ex, model, prompt, seq):
    """Every token behind the prompt is the largest logit's, as one call over the whole sequence computes them.
    Tokens may differ where two logits are nearer than the two computations: codes of a cache that was
    filled in other pieces differ in subnormals, queries and outputs are rounded to bf16 (2^-8 of a
    value), so a logit, a sum of 256 terms of variance 1/256, moves by about 2^-8; 0.05 is twelve of them."""
    tables, cache = ex.new_cache(model, 1, 8, 8)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    worst = 0.0
    for lo in range(0, len(seq) - 1, 128):
        part = seq[lo:min(lo + 128, len(seq) - 1)]
        q_start, kv_len, _, _ = tables.advance(i32([lo]), i32([len(part)]), len(part))
        logits = model(cache, torch.tensor(part, device="cuda"), q_start, kv_len)
        for i in range(len(part)):
            if lo + i + 1 >= len(prompt):
                worst = max(worst, (logits[i].max() - logits[i, seq[lo + i + 1]]).item())
    assert worst <= 0.05, worst


# (four blocks: the first three requests end with 2, 1 and 2, so that a place waits)
@pytest.mark.parametrize("n_blocks", [24, 4])
@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 8, 64)])
def test_drafts_do_not_change_what_is_decoded(ex, heads, n_blocks):
    model = ex.Model(n_q=heads[0], n_kv=heads[1], d_h=heads[2])
    prompts = prompts_of(model.vocab, (40, 3, 64, 25, 120, 1), 1)
    new = 40
    plain, a = ex.serve(model, prompts, new, lambda request, seq: [], n_blocks=n_blocks)
    rng = random.Random(2)

    def guess(request, seq):
        right = plain[request][len(seq):len(seq) + rng.randrange(6)]
        return [t if rng.random() < 0.7 else rng.randrange(model.vocab) for t in right]

    drafted, b = ex.serve(model, prompts, new, guess, n_blocks=n_blocks)
    for seqs in (plain, drafted):
        for p, s in zip(prompts, seqs):
            assert s[:len(p)] == p and len(s) == len(p) + new
            check_greedy(ex, model, p, s)
    assert 0 < b["kept"] < b["drafted"] and b["steps"] < a["steps"]
    assert (a["waited"] > 0) == (n_blocks == 4)
    capi.pipo_op_paged_check()


def test_drafts_at_a_temperature(ex):
    model = ex.Model()
    prompts = prompts_of(model.vocab, (30, 70), 3)
    seqs, c = ex.serve(model, prompts, 25, lambda request, seq: [seq[-1], seq[0], 5], temperature=1.0)
    assert all(len(s) == len(p) + 25 and all(0 <= t < model.vocab for t in s) for p, s in zip(prompts, seqs))
    again, _ = ex.serve(model, prompts, 25, lambda request, seq: [seq[-1], seq[0], 5], temperature=1.0)
    assert seqs == again


def test_a_step_in_one_graph():
    """Tables, append, attention and verification captured together; replays follow lengths, tokens and random
    numbers, beside eager calls of the same objects."""
    batch, n_q, n_kv, d, vocab, wide = 4, 8, 2, 64, 100, 4
    g = torch.Generator(device="cuda").manual_seed(4)
    pool = lambda: torch.zeros(40, n_kv, 64, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.ones(40, n_kv, device="cuda")  # noqa: E731
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731

    class Side:
        def __init__(self):
            self.tables = paged.BlockTables.new(batch, 10, 40)
            self.cache = paged.PagedCache8(pool(), pool(), scale(), scale(), self.tables.table, n_q=n_q)

        def step(self, kept, added, qkv, target, drafted, start, u, r):
            q_start, kv_len, slots, _ = self.tables.advance(kept, added, qkv.shape[0])
            q = self.cache.append(qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:], q_start, kv_len)
            o = self.cache.attend(q, q_start, kv_len)
            tokens, count = drafts.verify(target, drafted, start, u, r, width=wide)
            kept.add_(count)
            return o, tokens, count, slots, kv_len

    rows = batch * wide

    def inputs(seed):
        gg = torch.Generator(device="cuda").manual_seed(seed)
        start = torch.arange(batch + 1, dtype=torch.int32, device="cuda") * (wide - 1)
        return [torch.randn(rows, n_q + 2 * n_kv, d, generator=gg, device="cuda"),
                torch.softmax(torch.randn(rows, vocab, generator=gg, device="cuda") * 2, -1),
                torch.randint(0, 8, (batch * (wide - 1),), generator=gg, device="cuda", dtype=torch.int32), start,
                torch.rand(batch * (wide - 1), generator=gg, device="cuda") * 0.02,
                torch.rand(batch, generator=gg, device="cuda")]

    added = torch.full((batch,), wide, dtype=torch.int32, device="cuda")
    eager, captured = Side(), Side()
    kept = [torch.zeros(batch, dtype=torch.int32, device="cuda") for _ in range(2)]
    static = inputs(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        Side().step(torch.zeros_like(kept[0]), added, *static)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = captured.step(kept[1], added, *static)
    for i in range(12):
        now = inputs(i)
        for a, b in zip(static, now):
            a.copy_(b)
        graph.replay()
        want = eager.step(kept[0], added, *now)
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        assert torch.equal(kept[0], kept[1])
    assert kept[0].min() >= 12 and kept[0].max() > 12
