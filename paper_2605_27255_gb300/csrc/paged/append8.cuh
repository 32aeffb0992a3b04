// Norm, rotation and append of the new tokens to a cache of e4m3 codes.
//
// As append.cuh, but keys and values become codes: all new keys (or values) of a block and kv
// head are held in registers by one CTA, their largest magnitude sets the
// scale, and they are rounded once.  A block's first entry (slot 0 among the new ones)
// starts a new scale.  Later entries keep it while they fit (up to 448 times the scale);
// else it is chosen anew from them, and the codes that the block holds move by the
// ratio, a power of two.  It never falls: where the chosen one, capped at 2^7, would be below that of a pool
// which something else has filled, that one stays, new entries beyond it saturate, and no held code is touched.
//
// Bound by HBM: every new value is read once and written once.
#pragma once

#include <cuda_fp16.h>

#include "append.cuh"
#include "codes.cuh"

namespace pipo {

// the codes of slots 0 .. n-1 of a block's head, times `f`
template <int DH>
__device__ __forceinline__ void move_codes(uint8_t* block, int n, float f) {
    for (int i = threadIdx.x; i < n * (DH / 16); i += kAppendWarps * 32) {
        uint4 x = reinterpret_cast<uint4*>(block)[i];
        uint32_t* w = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = decode_lo(w[k]), hi = decode_hi(w[k]);
            const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
            const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
            w[k] = encode4(a.x * f, a.y * f, b.x * f, b.y * f);
        }
        reinterpret_cast<uint4*>(block)[i] = x;
    }
}

// grid: CTAs of kAppendWarps tokens' queries each, then page_ctas = runs * n_kv * 2 of (page, kv head, keys or
// values).  Keys and values apart, so that 64 registers hold a block's entries and four CTAs fit an SM: two
// 8191-token prompts with 32 query and 8 kv heads of 128 in bf16 117 us with both in one CTA (128 registers, two
// CTAs), 81 apart, 78 with the queries first (the other order ends in a tail of long CTAs), 72.4 now.
template <int DH, typename TI>
__global__ void __launch_bounds__(kAppendWarps * 32, 4) kv_append8_kernel(AppendArgs p, int page_ctas) {
    using HL = HeadLane<DH>;
    constexpr int E = kAppendWarps * HL::H, R = kPage / E;  // entries a round, rounds
    __shared__ float most[kAppendWarps];
    const PagedArgs& c = p.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = HL::dim(), hl = HL::head();
    pdl_launch();
    pdl_wait();
    float gain[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    const int query_ctas = (int)gridDim.x - page_ctas, x0 = (int)blockIdx.x - query_ctas;
    // Queries: a warp per token, the text of kv_append_kernel's (as a function that both call it compiles to a slower
    // schedule in either: 78 against 72.5 us there, 77 against 72.4 here)
    if (x0 < 0) {
        const long long t = (long long)blockIdx.x * kAppendWarps + warp;
        if (t >= c.n_tokens) return;
        load_gain<DH, bf16_t>(static_cast<const bf16_t*>(p.q_gain), gain);
        const Tok k = find_token(c, (int)t);
        if (k.b < 0) return;
        const Angles an = load_angles<DH>(k.pos >= 0 ? p.rope : nullptr, k.pos);
        const TI* src = static_cast<const TI*>(p.q) + (size_t)t * p.ld_q + d;
        bf16_t* dst = static_cast<bf16_t*>(p.q_out) + (size_t)t * c.n_q * DH + d;
        const float eps = k.pos >= 0 ? p.eps : 1.f;  // (a token without an entry: zeros, also where eps is 0)
        constexpr int U = 4;  // heads in flight per lane
        for (int h0 = 0; h0 < c.n_q; h0 += U * HL::H) {
            float a[U][4], b[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * HL::H + hl;
#pragma unroll
                for (int i = 0; i < 4; ++i) a[u][i] = b[u][i] = 0.f;
                if (h < c.n_q && k.pos >= 0) {
                    load_f<TI, 4>(src + (size_t)h * DH, a[u]);
                    load_f<TI, 4>(src + (size_t)h * DH + DH / 2, b[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * HL::H + hl;
                norm_turn<DH>(a[u], b[u], p.q_gain != nullptr, gain, eps, an);
                if (h < c.n_q) {
                    store_f<bf16_t, 4>(dst + (size_t)h * DH, a[u]);
                    store_f<bf16_t, 4>(dst + (size_t)h * DH + DH / 2, b[u]);
                }
            }
        }
        return;
    }
    const bool keys = (x0 & 1) == 0;
    const int g = x0 / 2 % c.n_kv;
    int b, page;
    if (!find_run(c, x0 / 2 / c.n_kv, b, page)) return;
    const int len = seq_len(c, b), end = q_row(c, b + 1), n = end - q_row(c, b);
    const int j0 = max(page * kPage, len - n), j1 = min(len, (page + 1) * kPage);  // the new entries
    const int blk = c.table[(size_t)b * c.max_pages + page];
    if (blk < 0 || blk >= c.n_blocks) return;
    const size_t head = (size_t)blk * c.n_kv + g;
    float* scale = (keys ? p.k_scale : p.v_scale) + head;
    const float old = *scale;
    const long long ld = keys ? p.ld_k : p.ld_v;
    const TI* src = static_cast<const TI*>(keys ? p.kn : p.vn) + (size_t)g * DH + d;
    float x[R][4], y[R][4];  // dims d .. and DH / 2 + d ..
    const int at = warp * HL::H + hl;  // this lane's entry of a round
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = j0 + r * E + at;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[r][i] = y[r][i] = 0.f;
        if (j < j1) {
            const TI* s = src + (size_t)(end - (len - j)) * ld;
            load_f<TI, 4>(s, x[r]);
            load_f<TI, 4>(s + DH / 2, y[r]);
        }
    }
    if (keys && (p.k_gain || p.rope)) {  // (with neither nothing is touched: infinity times a sine of zero would be NaN)
        load_gain<DH, bf16_t>(static_cast<const bf16_t*>(p.k_gain), gain);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int j = j0 + r * E + at;
            if (j0 + r * E >= j1) break;  // (the same for every lane: the norm's shuffles need them all)
            const Angles an = load_angles<DH>(j < j1 ? p.rope : nullptr, j);
            norm_turn<DH>(x[r], y[r], p.k_gain != nullptr, gain, j < j1 ? p.eps : 1.f, an);
        }
    }
    float m = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(fabsf(x[r][i]), fabsf(y[r][i])));
    if (m > 3.402823466e38f) {  // an infinity (NaN is not seen): it does not count
        m = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = fmaxf(m, fmaxf(finite_abs(x[r][i]), finite_abs(y[r][i])));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) most[warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAppendWarps; ++w) m = fmaxf(m, most[w]);
    const int slot0 = j0 - page * kPage;  // entries held before
    const float now = slot0 == 0 ? scale_of(m) : m > kCodeMax * old ? fmaxf(scale_of(m), old) : old, f = 1.f / now;
    uint8_t* dst = static_cast<uint8_t*>(keys ? c.k : c.v) + head * kPage * DH;
    if (slot0 > 0 && now != old) move_codes<DH>(dst, slot0, old / now);
    if (threadIdx.x == 0) *scale = now;  // (every thread has read the old one before the barrier)
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = j0 + r * E + at;
        if (j >= j1) continue;
        uint8_t* o = dst + (size_t)(j % kPage) * DH + d;
        *reinterpret_cast<uint32_t*>(o) = encode4(x[r][0] * f, x[r][1] * f, x[r][2] * f, x[r][3] * f);
        *reinterpret_cast<uint32_t*>(o + DH / 2) = encode4(y[r][0] * f, y[r][1] * f, y[r][2] * f, y[r][3] * f);
    }
}

}  // namespace pipo
