// Attention over a paged cache, one warp per (token, query head): the simplest
// form, every product on the CUDA cores in fp32.
#pragma once

#include "paged.cuh"

namespace pipo {

template <int DH, typename T>
__global__ void __launch_bounds__(128) attn_plain_kernel(AttnPagedArgs a) {
    constexpr int N = DH / 32;
    const PagedArgs& c = a.c;
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int l = threadIdx.x & 31;
    if (w >= (long long)c.n_tokens * c.n_q) return;
    const int t = (int)(w / c.n_q), h = (int)(w % c.n_q), g = h / c.G;
    const Tok k = find_token(c, t);
    if (k.b < 0) return;
    float q[N], o[N] = {}, m = -INFINITY, sum = 0.f;
    load_f<T, N>(static_cast<const T*>(a.q) + (size_t)t * a.ld_q + (size_t)h * DH + l * N, q);
    const int first = a.window > 0 ? max(0, k.pos - a.window + 1) : 0;
    const int32_t* list = a.pages ? a.pages + ((size_t)t * c.n_kv + g) * a.n_top : nullptr;
    const int np = list ? a.n_top : k.pos / kPage + 1;
    for (int i = list ? 0 : first / kPage; k.pos >= 0 && i < np; ++i) {
        const int p = list ? list[i] : i;
        if (p < 0) break;
        const size_t off = block_off(c, page_block(c, k.b, p), g) + l * N;
        const int j0 = max(first, p * kPage), j1 = min(k.pos + 1, (p + 1) * kPage);
        for (int j = j0; j < j1; ++j) {
            float x[N], s = 0.f;
            load_f<T, N>(static_cast<const T*>(c.k) + off + (size_t)(j % kPage) * DH, x);
#pragma unroll
            for (int e = 0; e < N; ++e) s = fmaf(q[e], x[e], s);
            s = warp_sum(s) * a.scale;
            const float mn = fmaxf(m, s), corr = expf(m - mn), pr = expf(s - mn);
            load_f<T, N>(static_cast<const T*>(c.v) + off + (size_t)(j % kPage) * DH, x);
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = fmaf(pr, x[e], o[e] * corr);
            sum = fmaf(sum, corr, pr);
            m = mn;
        }
    }
    const float inv = sum > 0.f ? 1.0f / sum : 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] *= inv;
    store_f<T, N>(static_cast<T*>(a.out) + (size_t)t * a.ld_out + (size_t)h * DH + l * N, o);
}

}  // namespace pipo
