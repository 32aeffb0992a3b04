"""A one-layer model served with drafted tokens over an 8-bit paged cache.

Requests wait for a place in the batch; a step feeds every place its prompt, or its last token and
a few drafted ones behind it, all in one ragged batch:

    blocks, lengths, slots                BlockTables.advance
    qkv, norm, rotate, append             pipo_op_gemm_tc, PagedCache8.append
    attend to everything cached           PagedCache8.attend
    probabilities of the next tokens      pipo_op_gemm_tc, softmax
    keep drafts, draw one token more      drafts.verify

Entries of rejected drafts are given back by the next step's advance, like those of requests that
have ended; a request that the pool has no blocks for waits in its place.

Run on a GPU:  python examples/drafted_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paged_layer import PAGE, Layer, paged  # noqa: E402
from paper_2605_27255_gb300 import drafts  # noqa: E402


class WideLayer(Layer):
    """The layer for batches of any number of rows (a projection takes 128)."""

    @staticmethod
    def _project(W, x):
        return torch.cat([Layer._project(W, x[i:i + 128]) for i in range(0, x.shape[0], 128)])


class Model:
    """Random embeddings, one attention layer (paged_layer.py), its normalised output into a random head."""

    def __init__(self, vocab=512, hidden=256, n_q=8, n_kv=2, d_h=128, max_ctx=1024, seed=0):
        self.layer = WideLayer(hidden, n_q, n_kv, d_h, max_ctx, seed)
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.vocab = vocab
        self.embed = torch.randn(vocab, hidden, generator=g, device="cuda")
        self.head = (torch.randn(vocab, hidden, generator=g, device="cuda") / hidden ** 0.5).bfloat16()

    def __call__(self, cache, tokens, q_start, kv_len):
        """Logits [tokens, vocab] of a ragged batch, its entries appended."""
        y = self.layer(cache, self.embed[tokens], q_start, kv_len)
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True))
        return self.layer._project(self.head, y)


def new_cache(model, places, n_blocks, max_pages):
    """Empty tables, and a cache of codes under them."""
    tables = paged.BlockTables.new(places, max_pages, n_blocks)
    pool = lambda: torch.zeros(n_blocks, model.layer.n_kv, PAGE, model.layer.d_h, dtype=torch.uint8,  # noqa: E731
                               device="cuda").view(torch.float8_e4m3fn)
    scale = lambda: torch.ones(n_blocks, model.layer.n_kv, device="cuda")  # noqa: E731
    return tables, paged.PagedCache8(pool(), pool(), scale(), scale(), tables.table, n_q=model.layer.n_q)


def serve(model, prompts, new, guess, places=3, n_blocks=24, max_pages=8, temperature=0.0, seed=0):
    """Decodes `new` tokens for every prompt (a list of ids).  guess(request, tokens) names the drafted
    ids behind a request's tokens so far, which are taken as certain.  Returns the
    requests' tokens and counts of steps, drafted and kept tokens and of places that waited."""
    tables, cache = new_cache(model, places, n_blocks, max_pages)
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    waiting, seqs = list(range(len(prompts))), [list(p) for p in prompts]
    place, kept = [None] * places, [0] * places
    count = dict(steps=0, drafted=0, kept=0, waited=0)
    while waiting or any(p is not None for p in place):
        feed, first = [[] for _ in place], [0] * places  # tokens of a place, the first that is followed by a draft
        for b in range(places):
            if place[b] is None and waiting:
                place[b], kept[b] = waiting.pop(0), 0
            if place[b] is None:
                continue
            seq = seqs[place[b]]
            feed[b] = seq[kept[b]:]
            first[b] = len(feed[b]) - 1
            left = len(prompts[place[b]]) + new - len(seq)
            feed[b] += guess(place[b], seq)[:left - 1] if kept[b] else []
        q_start, kv_len, _, _ = tables.advance(i32(kept), i32([len(f) for f in feed]), sum(len(f) for f in feed))
        start = q_start.tolist()
        served = [b for b in range(places) if feed[b] and start[b + 1] > start[b]]
        count["steps"] += 1
        count["waited"] += sum(bool(f) for f in feed) - len(served)
        if not served:
            raise RuntimeError("the pool has too few blocks for any request")
        logits = model(cache, torch.tensor([t for b in served for t in feed[b]], device="cuda"), q_start, kv_len)
        rows = [start[b] + i for b in served for i in range(first[b], len(feed[b]))]
        target = logits[rows]
        if temperature > 0:
            target = torch.softmax(target / temperature, -1)
        else:
            target = torch.nn.functional.one_hot(target.argmax(-1), model.vocab).float()
        drafted = [feed[b][first[b] + 1:] for b in served]
        offsets = [0]
        for d in drafted:
            offsets.append(offsets[-1] + len(d))
        ids = i32([t for d in drafted for t in d])
        tokens, n = drafts.verify(target.contiguous(), ids, i32(offsets), torch.rand(len(ids), generator=g, device="cuda"),
                                  torch.rand(len(served), generator=g, device="cuda"), width=1 + max(map(len, drafted)))
        for b, row, k, d in zip(served, tokens.tolist(), n.tolist(), drafted):
            seqs[place[b]] += row[:k]
            # the fed tokens up to the last kept draft are cached, the drawn one is not
            kept[b] += first[b] + k
            count["drafted"] += len(d)
            count["kept"] += k - 1
            if len(seqs[place[b]]) >= len(prompts[place[b]]) + new:
                place[b], kept[b] = None, 0
    tables.advance(i32([0] * places), i32([0] * places), 0)
    assert int(tables.n_free) == n_blocks
    return seqs, count


def main():
    model = Model()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.vocab, (n,), generator=g).tolist() for n in (40, 3, 64, 25, 90)]
    plain, a = serve(model, prompts, 30, lambda request, seq: [])
    right = lambda request, seq: [t if i % 3 else (t + 1) % model.vocab  # noqa: E731
                                  for i, t in enumerate(plain[request][len(seq):len(seq) + 4], len(seq))]
    drafted, b = serve(model, prompts, 30, right)
    same = sum(x == y for p, q in zip(plain, drafted) for x, y in zip(p, q)) / sum(map(len, plain))
    print(f"one token a step: {a['steps']} steps; with drafts: {b['steps']} steps, {b['kept']} of {b['drafted']} kept; "
          f"{same:.1%} of the tokens are the same")


if __name__ == "__main__":
    main()
