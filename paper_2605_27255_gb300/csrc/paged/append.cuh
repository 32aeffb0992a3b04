// Norm, rotation and append of the new tokens' queries, keys and values.
//
//   q' = R(pos) r(q),  k' = R(pos) r(k),  r(x) = x / sqrt(mean(x^2) + eps) * gain
//
// per head in fp32, rounded once to the pools' type.  Bound by HBM: every value is
// read and written once.  DH / 8 lanes hold a head, each four dims of either half, so
// that the rotation's pairs are in one lane and every load and store is 8 or 16
// bytes; a warp holds 256 / DH heads at a time.
//
// A CTA takes either the new entries of one (page, kv head) (then nothing but this
// CTA writes that page's head, and the page's mean key needs no atomics and has
// a fixed order of addition), or all query heads of a few tokens, a warp per token: the
// token's angles and position are then looked up once.
#pragma once

#include "paged.cuh"

namespace pipo {

constexpr int kAppendWarps = 8;

// where a head's part of this lane lies
template <int DH>
struct HeadLane {
    static constexpr int L = DH / 8, H = 32 / L;  // lanes per head, heads per warp
    static __device__ __forceinline__ int dim() { return 4 * ((threadIdx.x & 31) % L); }
    static __device__ __forceinline__ int head() { return (threadIdx.x & 31) / L; }
};

// the angles of this lane's four pairs
struct Angles {
    float c[4], s[4];
};
template <int DH>
__device__ __forceinline__ Angles load_angles(const float* rope, int pos) {
    Angles a;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a.c[i] = 1.f;
        a.s[i] = 0.f;
    }
    if (rope) {
        const float4* r = reinterpret_cast<const float4*>(rope + (size_t)pos * DH + 2 * HeadLane<DH>::dim());
        const float4 x = r[0], y = r[1];
        a.c[0] = x.x; a.s[0] = x.y; a.c[1] = x.z; a.s[1] = x.w;
        a.c[2] = y.x; a.s[2] = y.y; a.c[3] = y.z; a.s[3] = y.w;
    }
    return a;
}

// gains of this lane's dims (both halves)
template <int DH, typename T>
__device__ __forceinline__ void load_gain(const T* gain, float (&g)[8]) {
    if (!gain) return;
    const int d = HeadLane<DH>::dim();
    float a[4], b[4];
    load_f<T, 4>(gain + d, a);
    load_f<T, 4>(gain + DH / 2 + d, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = a[i];
        g[4 + i] = b[i];
    }
}

// this lane's part of a head, normalised and rotated in place (every lane of the head calls it)
template <int DH>
__device__ __forceinline__ void norm_turn(float (&a)[4], float (&b)[4], bool norm, const float (&g)[8], float eps,
                                          const Angles& an) {
    if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) ss += a[i] * a[i] + b[i] * b[i];
#pragma unroll
        for (int o = HeadLane<DH>::L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float r = 1.0f / sqrtf(ss * (1.0f / DH) + eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] *= r * g[i];
            b[i] *= r * g[4 + i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float x = a[i], y = b[i];
        a[i] = x * an.c[i] - y * an.s[i];
        b[i] = y * an.c[i] + x * an.s[i];
    }
}

// The r-th (sequence, page) that receives entries, in order: false when there
// are fewer.  Every thread of a warp gets the same answer.
__device__ __forceinline__ bool find_run(const PagedArgs& c, int r, int& b, int& page) {
    const int lane = threadIdx.x & 31;
    for (int b0 = 0; b0 < c.batch; b0 += 32) {
        int n = 0, first = 0;
        if (b0 + lane < c.batch) {
            const int len = seq_len(c, b0 + lane);
            const int p0 = max(0, len - max(0, q_row(c, b0 + lane + 1) - q_row(c, b0 + lane)));
            first = p0 / kPage;
            if (p0 < len) n = (len - 1) / kPage - first + 1;
        }
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, r >= incl - n && r < incl);
        if (hit) {
            const int src = __ffs(hit) - 1;
            b = b0 + src;
            page = __shfl_sync(0xffffffffu, first + r - (incl - n), src);
            return true;
        }
        r -= __shfl_sync(0xffffffffu, incl, 31);
    }
    return false;
}

// Four CTAs an SM (64 registers) keep enough loads in flight: 74 us for two 8191-token prompts,
// 5.6 TB/s; with two entries per lane at a time 80, with the registers that take (three CTAs) 89, with 16
// dims per lane 90.
// grid: page_ctas = runs * n_kv CTAs of (page, kv head), then kAppendWarps tokens' queries each
template <int DH, typename TI, typename T>
__global__ void __launch_bounds__(kAppendWarps * 32, 4) kv_append_kernel(AppendArgs p, int page_ctas) {
    using HL = HeadLane<DH>;
    __shared__ float acc[kAppendWarps][HL::H][DH];
    const PagedArgs& c = p.c;
    const int warp = threadIdx.x >> 5, d = HL::dim(), hl = HL::head();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float gain[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if ((int)blockIdx.x >= page_ctas) {  // queries: a warp per token
        const long long t = ((long long)blockIdx.x - page_ctas) * kAppendWarps + warp;
        if (t >= c.n_tokens) return;
        load_gain<DH, T>(static_cast<const T*>(p.q_gain), gain);
        const Tok k = find_token(c, (int)t);
        if (k.b < 0) return;
        const Angles an = load_angles<DH>(k.pos >= 0 ? p.rope : nullptr, k.pos);
        const TI* src = static_cast<const TI*>(p.q) + (size_t)t * p.ld_q + d;
        T* dst = static_cast<T*>(p.q_out) + (size_t)t * c.n_q * DH + d;
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
                    store_f<T, 4>(dst + (size_t)h * DH, a[u]);
                    store_f<T, 4>(dst + (size_t)h * DH + DH / 2, b[u]);
                }
            }
        }
        return;
    }
    const int g = blockIdx.x % c.n_kv;
    int b, page;
    if (!find_run(c, blockIdx.x / c.n_kv, b, page)) return;
    const int len = seq_len(c, b), end = q_row(c, b + 1), n = end - q_row(c, b);
    const int j0 = max(page * kPage, len - n), j1 = min(len, (page + 1) * kPage);  // the new entries
    const int blk = c.table[(size_t)b * c.max_pages + page];
    if (blk < 0 || blk >= c.n_blocks) return;
    load_gain<DH, T>(static_cast<const T*>(p.k_gain), gain);
    T* kd = static_cast<T*>(c.k) + block_off(c, blk, g) + d;
    T* vd = static_cast<T*>(c.v) + block_off(c, blk, g) + d;
    float sa[4] = {}, sb[4] = {};  // this lane's part of the page's sum
    for (int jj = j0; jj < j1; jj += kAppendWarps * HL::H) {
        const int j = jj + warp * HL::H + hl;
        const Angles an = load_angles<DH>(j < j1 ? p.rope : nullptr, j);
        float a[4] = {}, bb[4] = {}, va[4] = {}, vb[4] = {};
        if (j < j1) {
            const size_t t = (size_t)(end - (len - j));
            const TI* ks = static_cast<const TI*>(p.kn) + t * p.ld_k + (size_t)g * DH + d;
            const TI* vs = static_cast<const TI*>(p.vn) + t * p.ld_v + (size_t)g * DH + d;
            load_f<TI, 4>(ks, a);
            load_f<TI, 4>(ks + DH / 2, bb);
            load_f<TI, 4>(vs, va);
            load_f<TI, 4>(vs + DH / 2, vb);
        }
        norm_turn<DH>(a, bb, p.k_gain != nullptr, gain, p.eps, an);
        if (j < j1) {
            const size_t o = (size_t)(j % kPage) * DH;
            store_f<T, 4>(kd + o, a);
            store_f<T, 4>(kd + o + DH / 2, bb);
            store_f<T, 4>(vd + o, va);
            store_f<T, 4>(vd + o + DH / 2, vb);
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // the mean is of the keys as stored
                sa[i] += to_f(from_f<T>(a[i]));
                sb[i] += to_f(from_f<T>(bb[i]));
            }
        }
    }
    if (!c.means) return;
#pragma unroll 4
    for (int j = page * kPage + warp * HL::H + hl; j < j0; j += kAppendWarps * HL::H) {  // the entries it held before
        float a[4], bb[4];
        load_f<T, 4>(kd + (size_t)(j % kPage) * DH, a);
        load_f<T, 4>(kd + (size_t)(j % kPage) * DH + DH / 2, bb);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sa[i] += a[i];
            sb[i] += bb[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        acc[warp][hl][d + i] = sa[i];
        acc[warp][hl][DH / 2 + d + i] = sb[i];
    }
    __syncthreads();
    if (threadIdx.x < DH) {
        float s = 0.f;
        for (int w = 0; w < kAppendWarps; ++w)
            for (int h = 0; h < HL::H; ++h) s += acc[w][h][threadIdx.x];
        static_cast<T*>(c.means)[((size_t)blk * c.n_kv + g) * DH + threadIdx.x] = from_f<T>(s / (float)(j1 - page * kPage));
    }
}

}  // namespace pipo
