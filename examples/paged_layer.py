"""One GQA attention layer over a paged cache, served with continuous batching.

Three requests with prompts of different lengths share one cache.  A call takes
at most 128 tokens: prompts come in chunks while requests that have finished
theirs decode one token a call, all in the same ragged batch.  The layer is

    qkv = Wqkv . x                       pipo_op_gemm_tc (tcgen05)
    norm, rotate, append                 PagedCache.append
    attend to everything cached          PagedCache.attend
    or score the pages, attend to a few  PagedCache.page_scores, attend_pages
    y = Wo . o                           pipo_op_gemm_tc

Run on a GPU:  python examples/paged_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_27255_gb300 import capi, paged  # noqa: E402

PAGE = paged.PAGE


class Layer:
    """Random weights at the 4B model's head shape (32 query and 8 kv heads of
    128, with per-head norms of queries and keys) behind a hidden size of 1024."""

    def __init__(self, hidden=1024, n_q=32, n_kv=8, d_h=128, max_ctx=4096, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device=device) * 0.02).to(torch.bfloat16)  # noqa: E731
        self.hidden, self.n_q, self.n_kv, self.d_h = hidden, n_q, n_kv, d_h
        self.Wqkv, self.Wo = w((n_q + 2 * n_kv) * d_h, hidden), w(hidden, n_q * d_h)
        self.q_gain = (1 + 5 * w(d_h).float()).to(torch.bfloat16)
        self.k_gain = (1 + 5 * w(d_h).float()).to(torch.bfloat16)
        self.rope = paged.rope_table(max_ctx, d_h, 1.0e6, device)

    @staticmethod
    def _project(W, x):
        """W . x for up to 128 rows of fp32 activations."""
        y = torch.empty(x.shape[0], W.shape[0], device=x.device)
        need = capi.pipo_op_gemm_tc_scratch(0, W.shape[0], W.shape[1], x.shape[0])
        buf = torch.empty(need + 1024, dtype=torch.uint8, device=x.device)
        at = -buf.data_ptr() % 1024
        capi.pipo_op_gemm_tc(0, W.data_ptr(), W.shape[0], W.shape[1], x.data_ptr(), x.shape[0], y.data_ptr(), 0,
                             buf.data_ptr() + at, need, torch.cuda.current_stream().cuda_stream)
        return y

    def __call__(self, cache, x, q_start, kv_len, top=0):
        """x: fp32 [tokens, hidden] of the batch; top > 0: that many pages per token and kv head."""
        qkv = self._project(self.Wqkv, x).view(x.shape[0], -1, self.d_h)
        q, k, v = qkv.split([self.n_q, self.n_kv, self.n_kv], 1)
        q = cache.append(q, k, v, q_start, kv_len, q_gain=self.q_gain, k_gain=self.k_gain, rope=self.rope)
        if top:
            o, _ = cache.attend_pages(q, cache.page_scores(q, q_start, kv_len), q_start, kv_len, top=top, sink=1,
                                      local=2)
        else:
            o = cache.attend(q, q_start, kv_len)
        return self._project(self.Wo, o.float().view(x.shape[0], -1))


def new_cache(layer, requests, max_ctx=4096, device="cuda"):
    """Pools with a block for every page of every request, in a random order."""
    width = max_ctx // PAGE
    blocks = requests * width
    pool = lambda: torch.zeros(blocks, layer.n_kv, PAGE, layer.d_h, dtype=torch.bfloat16, device=device)  # noqa: E731
    g = torch.Generator().manual_seed(1)
    table = torch.randperm(blocks, generator=g).view(requests, width).to(torch.int32).to(device)
    means = torch.zeros(blocks, layer.n_kv, layer.d_h, dtype=torch.bfloat16, device=device)
    return paged.PagedCache(pool(), pool(), table, n_q=layer.n_q, means=means)


def serve(layer, inputs, budget=128, top=0):
    """Feeds every request's rows (prompt and decoded tokens, fp32
    [tokens, hidden]) through the layer: whatever is left of the prompts in chunks of at most
    `budget` rows a call, shared evenly, one row at least for each request that
    has any left.  Returns every request's outputs."""
    cache = new_cache(layer, len(inputs))
    done = [0] * len(inputs)
    out = [[] for _ in inputs]
    while any(d < x.shape[0] for d, x in zip(done, inputs)):
        live = [b for b, x in enumerate(inputs) if done[b] < x.shape[0]]
        take = [min(inputs[b].shape[0] - done[b], max(1, budget // len(live))) if b in live else 0
                for b in range(len(inputs))]
        rows = torch.cat([x[d:d + n] for x, d, n in zip(inputs, done, take)])
        done = [d + n for d, n in zip(done, take)]
        start = [0]
        for n in take:
            start.append(start[-1] + n)
        y = layer(cache, rows, torch.tensor(start, dtype=torch.int32, device=rows.device),
                  torch.tensor(done, dtype=torch.int32, device=rows.device), top)
        for b, n in enumerate(take):
            if n:
                out[b].append(y[start[b]:start[b] + n])
    capi.pipo_op_paged_check()
    return [torch.cat(o) for o in out]


def main():
    layer = Layer()
    g = torch.Generator(device="cuda").manual_seed(2)
    inputs = [torch.randn(n, layer.hidden, generator=g, device="cuda") for n in (1000, 77, 300)]
    mixed = serve(layer, inputs)
    alone = [serve(layer, [x])[0] for x in inputs]
    few = serve(layer, inputs, top=6)
    for b, (m, a, f) in enumerate(zip(mixed, alone, few)):
        print(f"request {b}: {m.shape[0]} tokens; batched against alone: largest difference "
              f"{(m - a).abs().max().item():.2e} of {a.abs().max().item():.2e}; six pages a token: "
              f"{((f - m).norm() / m.norm()).item():.3f} of the norm away")


if __name__ == "__main__":
    main()
