// Norm, rotation and append of the new tokens to a cache of e4m3 codes.
//
// As append.cuh, but keys and values become codes: of a block and kv head all new
// entries are held in registers by one CTA, their largest magnitude sets the
// scale, and they are rounded once.  A block's first entry (slot 0 among the new ones)
// starts a new scale.  Later entries keep it while they fit (up to 448 times the scale);
// else it is chosen anew from them, and the codes that the block holds move by the
// ratio, a power of two.
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

// grid: page_ctas = runs * n_kv CTAs of (page, kv head), then kAppendWarps tokens' queries each
template <int DH, typename TI>
__global__ void __launch_bounds__(kAppendWarps * 32, 2) kv_append8_kernel(AppendArgs p, int page_ctas) {
    using HL = HeadLane<DH>;
    constexpr int E = kAppendWarps * HL::H, R = kPage / E;  // entries a round, rounds
    __shared__ float most[2][kAppendWarps];
    const PagedArgs& c = p.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = HL::dim(), hl = HL::head();
    pdl_launch();
    pdl_wait();
    if ((int)blockIdx.x >= page_ctas) {
        append_queries<DH, TI, bf16_t>(p, ((long long)blockIdx.x - page_ctas) * kAppendWarps + warp);
        return;
    }
    const int g = blockIdx.x % c.n_kv;
    int b, page;
    if (!find_run(c, blockIdx.x / c.n_kv, b, page)) return;
    const int len = seq_len(c, b), end = q_row(c, b + 1), n = end - q_row(c, b);
    const int j0 = max(page * kPage, len - n), j1 = min(len, (page + 1) * kPage);  // the new entries
    const int blk = c.table[(size_t)b * c.max_pages + page];
    if (blk < 0 || blk >= c.n_blocks) return;
    const size_t head = (size_t)blk * c.n_kv + g;
    const float old_k = p.k_scale[head], old_v = p.v_scale[head];
    float gain[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    load_gain<DH, bf16_t>(static_cast<const bf16_t*>(p.k_gain), gain);
    float ka[R][4], kb[R][4], va[R][4], vb[R][4];
    const int at = warp * HL::H + hl;  // this lane's entry of a round
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = j0 + r * E + at;
#pragma unroll
        for (int i = 0; i < 4; ++i) ka[r][i] = kb[r][i] = va[r][i] = vb[r][i] = 0.f;
        if (j < j1) {
            const size_t t = (size_t)(end - (len - j));
            const TI* ks = static_cast<const TI*>(p.kn) + t * p.ld_k + (size_t)g * DH + d;
            const TI* vs = static_cast<const TI*>(p.vn) + t * p.ld_v + (size_t)g * DH + d;
            load_f<TI, 4>(ks, ka[r]);
            load_f<TI, 4>(ks + DH / 2, kb[r]);
            load_f<TI, 4>(vs, va[r]);
            load_f<TI, 4>(vs + DH / 2, vb[r]);
        }
    }
    float mk = 0.f, mv = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = j0 + r * E + at;
        if (j0 + r * E >= j1) break;  // (the same for every lane: the norm's shuffles need them all)
        const Angles an = load_angles<DH>(j < j1 ? p.rope : nullptr, j);
        // (without angles nothing is turned: infinity times a sine of zero would be NaN in its partner)
        norm_turn<DH>(ka[r], kb[r], p.k_gain != nullptr, gain, j < j1 ? p.eps : 1.f, an, p.rope != nullptr);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mk = fmaxf(mk, fmaxf(finite_abs(ka[r][i]), finite_abs(kb[r][i])));
            mv = fmaxf(mv, fmaxf(finite_abs(va[r][i]), finite_abs(vb[r][i])));
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mk = fmaxf(mk, __shfl_xor_sync(0xffffffffu, mk, o));
        mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, o));
    }
    if (lane == 0) {
        most[0][warp] = mk;
        most[1][warp] = mv;
    }
    __syncthreads();
    mk = mv = 0.f;
#pragma unroll
    for (int w = 0; w < kAppendWarps; ++w) {
        mk = fmaxf(mk, most[0][w]);
        mv = fmaxf(mv, most[1][w]);
    }
    const int slot0 = j0 - page * kPage;  // entries held before
    const float new_k = slot0 == 0 || mk > kCodeMax * old_k ? scale_of(mk) : old_k;
    const float new_v = slot0 == 0 || mv > kCodeMax * old_v ? scale_of(mv) : old_v;
    uint8_t* kd = static_cast<uint8_t*>(c.k) + head * kPage * DH;
    uint8_t* vd = static_cast<uint8_t*>(c.v) + head * kPage * DH;
    if (slot0 > 0 && new_k != old_k) move_codes<DH>(kd, slot0, old_k / new_k);
    if (slot0 > 0 && new_v != old_v) move_codes<DH>(vd, slot0, old_v / new_v);
    if (threadIdx.x == 0) {  // (every thread has read the old ones before the barrier)
        p.k_scale[head] = new_k;
        p.v_scale[head] = new_v;
    }
    const float fk = 1.f / new_k, fv = 1.f / new_v;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = j0 + r * E + at;
        if (j >= j1) continue;
        const size_t o = (size_t)(j % kPage) * DH + d;
        *reinterpret_cast<uint32_t*>(kd + o) = encode4(ka[r][0] * fk, ka[r][1] * fk, ka[r][2] * fk, ka[r][3] * fk);
        *reinterpret_cast<uint32_t*>(kd + o + DH / 2) = encode4(kb[r][0] * fk, kb[r][1] * fk, kb[r][2] * fk, kb[r][3] * fk);
        *reinterpret_cast<uint32_t*>(vd + o) = encode4(va[r][0] * fv, va[r][1] * fv, va[r][2] * fv, va[r][3] * fv);
        *reinterpret_cast<uint32_t*>(vd + o + DH / 2) = encode4(vb[r][0] * fv, vb[r][1] * fv, vb[r][2] * fv, vb[r][3] * fv);
    }
}

}  // namespace pipo
