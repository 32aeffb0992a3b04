// Page scores and the selection of pages.
#pragma once

#include "paged.cuh"

namespace pipo {

// scores[t][g][p] = scale * sum_h q[t, h] . mean[p]; one warp per (token, kv head)
template <int DH, typename T>
__global__ void __launch_bounds__(128) page_scores_kernel(ScoreArgs a) {
    constexpr int N = DH / 32;
    const PagedArgs& c = a.c;
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int l = threadIdx.x & 31;
    if (w >= (long long)c.n_tokens * c.n_kv) return;
    const int t = (int)(w / c.n_kv), g = (int)(w % c.n_kv);
    const Tok k = find_token(c, t);
    if (k.b < 0) return;
    float q[N] = {};
    for (int h = 0; h < c.G; ++h) {
        float x[N];
        load_f<T, N>(static_cast<const T*>(a.q) + (size_t)t * a.ld_q + (size_t)(g * c.G + h) * DH + l * N, x);
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] += x[i];
    }
    const int seen = k.pos < 0 ? 0 : k.pos / kPage + 1;
    float* o = a.scores + (size_t)w * c.max_pages;
    for (int p = 0; p < seen; ++p) {
        float x[N], s = 0.f;
        load_f<T, N>(static_cast<const T*>(c.means) + ((size_t)page_block(c, k.b, p) * c.n_kv + g) * DH + l * N, x);
#pragma unroll
        for (int i = 0; i < N; ++i) s = fmaf(q[i], x[i], s);
        s = warp_sum(s);
        if (l == 0) o[p] = s * a.scale;
    }
    for (int p = seen + l; p < c.max_pages; p += 32) o[p] = -INFINITY;
}

// Scores as integers of the same order: NaN lowest, the two zeros alike.
__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Kept pages of one (token, kv head) per warp: the pages that have to be
// kept, then the n_top - (those) largest keys, found bit by bit (the largest
// key that at least so many reach), equal keys from the lowest page on.
__global__ void __launch_bounds__(128) page_select_kernel(SelectArgs a) {
    const PagedArgs& c = a.c;
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int l = threadIdx.x & 31;
    if (w >= (long long)c.n_tokens * c.n_kv) return;
    const Tok k = find_token(c, (int)(w / c.n_kv));
    if (k.b < 0) return;
    int32_t* o = a.pages + (size_t)w * a.n_top;
    const float* sc = a.scores + (size_t)w * c.max_pages;
    const int seen = k.pos < 0 ? 0 : k.pos / kPage + 1;
    const int head = min(a.n_sink, seen), tail = max(head, seen - a.n_local);  // candidates: [head, tail)
    int want = min(a.n_top, seen) - (seen - tail + head);                       // of them to be kept
    uint32_t key = 0;
    if (want < tail - head) {
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t trial = key | (1u << bit);
            int n = 0;
            for (int p = head + l; p < tail; p += 32) n += score_key(sc[p]) >= trial;
            if ((int)__reduce_add_sync(0xffffffffu, n) >= want) key = trial;
        }
    }
    int above = 0;  // keys above the last one kept
    for (int p = head + l; p < tail; p += 32) above += score_key(sc[p]) > key;
    int ties = want - (int)__reduce_add_sync(0xffffffffu, above);
    int n = 0;
    for (int p0 = 0; p0 < seen; p0 += 32) {
        const int p = p0 + l;
        const bool cand = p >= head && p < tail;
        const uint32_t x = cand ? score_key(sc[p]) : 0u;
        const unsigned eq = __ballot_sync(0xffffffffu, cand && x == key);
        const bool keep = p < seen && (!cand || x > key || (x == key && __popc(eq & ((1u << l) - 1u)) < ties));
        const unsigned kept = __ballot_sync(0xffffffffu, keep);
        if (keep) o[n + __popc(kept & ((1u << l) - 1u))] = p;
        n += __popc(kept);
        ties -= min(ties, (int)__popc(eq));
    }
    for (int i = n + l; i < a.n_top; i += 32) o[i] = -1;
}

}  // namespace pipo
