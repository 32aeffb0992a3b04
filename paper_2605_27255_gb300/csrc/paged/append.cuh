// Norm, rotation and append of the new tokens' queries, keys and values.
//
//   q' = R(pos) r(q),  k' = R(pos) r(k),  r(x) = x / sqrt(mean(x^2) + eps) * gain
//
// per head in fp32, rounded once to the pools' type.  A CTA takes either the
// new entries of one (page, kv head) (then nothing but this CTA writes that
// page's head, and the page's mean key needs no atomics), or a group of query
// rows.  A warp holds one head at a time: lane l the dims that start at l * DH/64
// of both halves, so that the rotation's pairs are in one lane.
#pragma once

#include "paged.cuh"

namespace pipo {

constexpr int kAppendWarps = 8;
constexpr int kAppendRows = 4;  // query rows per warp

// this lane's part of one head, normalised and rotated
template <int DH, typename TI, typename T>
__device__ __forceinline__ void head_in(const TI* x, const T* gain, const float* rope, float eps, float (&a)[DH / 64],
                                        float (&b)[DH / 64]) {
    constexpr int N = DH / 64;
    const int l = threadIdx.x & 31;
    load_f<TI, N>(x + l * N, a);
    load_f<TI, N>(x + DH / 2 + l * N, b);
    if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) ss += a[i] * a[i] + b[i] * b[i];
        const float r = 1.0f / sqrtf(warp_sum(ss) * (1.0f / DH) + eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] *= r * to_f(gain[l * N + i]);
            b[i] *= r * to_f(gain[DH / 2 + l * N + i]);
        }
    }
    if (rope) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float c = rope[2 * (l * N + i)], s = rope[2 * (l * N + i) + 1], x1 = a[i], x2 = b[i];
            a[i] = x1 * c - x2 * s;
            b[i] = x2 * c + x1 * s;
        }
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

// grid: page_ctas = runs * n_kv CTAs of (page, kv head), then the query rows
template <int DH, typename TI, typename T>
__global__ void __launch_bounds__(kAppendWarps * 32) kv_append_kernel(AppendArgs p, int page_ctas) {
    constexpr int N = DH / 64;
    __shared__ float acc[kAppendWarps][DH];
    const PagedArgs& c = p.c;
    const int warp = threadIdx.x >> 5, l = threadIdx.x & 31;
    if ((int)blockIdx.x >= page_ctas) {  // queries
        const long long row0 = ((long long)blockIdx.x - page_ctas) * (kAppendWarps * kAppendRows) + warp * kAppendRows;
        for (int i = 0; i < kAppendRows; ++i) {
            const long long row = row0 + i;
            if (row >= (long long)c.n_tokens * c.n_q) return;
            const int t = (int)(row / c.n_q), h = (int)(row % c.n_q);
            const Tok k = find_token(c, t);
            if (k.b < 0) continue;
            float a[N] = {}, b[N] = {};
            if (k.pos >= 0)
                head_in<DH, TI, T>(static_cast<const TI*>(p.q) + (size_t)t * p.ld_q + (size_t)h * DH,
                                   static_cast<const T*>(p.q_gain), p.rope ? p.rope + (size_t)k.pos * DH : nullptr, p.eps,
                                   a, b);
            T* o = static_cast<T*>(p.q_out) + (size_t)row * DH + l * N;
            store_f<T, N>(o, a);
            store_f<T, N>(o + DH / 2, b);
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
    T* kd = static_cast<T*>(c.k) + block_off(c, blk, g);
    T* vd = static_cast<T*>(c.v) + block_off(c, blk, g);
    float sa[N] = {}, sb[N] = {};  // this warp's part of the page's sum
    for (int j = j0 + warp; j < j1; j += kAppendWarps) {
        const size_t t = (size_t)(end - (len - j));
        float a[N], bb[N];
        head_in<DH, TI, T>(static_cast<const TI*>(p.kn) + t * p.ld_k + (size_t)g * DH, static_cast<const T*>(p.k_gain),
                           p.rope ? p.rope + (size_t)j * DH : nullptr, p.eps, a, bb);
        T* o = kd + (size_t)(j % kPage) * DH + l * N;
        store_f<T, N>(o, a);
        store_f<T, N>(o + DH / 2, bb);
#pragma unroll
        for (int i = 0; i < N; ++i) {  // the mean is of the keys as stored
            sa[i] += to_f(from_f<T>(a[i]));
            sb[i] += to_f(from_f<T>(bb[i]));
        }
        const TI* vs = static_cast<const TI*>(p.vn) + t * p.ld_v + (size_t)g * DH;
        load_f<TI, N>(vs + l * N, a);
        load_f<TI, N>(vs + DH / 2 + l * N, bb);
        o = vd + (size_t)(j % kPage) * DH + l * N;
        store_f<T, N>(o, a);
        store_f<T, N>(o + DH / 2, bb);
    }
    if (!c.means) return;
    for (int j = page * kPage + warp; j < j0; j += kAppendWarps) {  // the entries it held before
        float a[N], bb[N];
        const T* o = kd + (size_t)(j % kPage) * DH + l * N;
        load_f<T, N>(o, a);
        load_f<T, N>(o + DH / 2, bb);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            sa[i] += a[i];
            sb[i] += bb[i];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        acc[warp][l * N + i] = sa[i];
        acc[warp][DH / 2 + l * N + i] = sb[i];
    }
    __syncthreads();
    if (threadIdx.x < DH) {
        float s = 0.f;
        for (int w = 0; w < kAppendWarps; ++w) s += acc[w][threadIdx.x];
        static_cast<T*>(c.means)[((size_t)blk * c.n_kv + g) * DH + threadIdx.x] = from_f<T>(s / (float)(j1 - page * kPage));
    }
}

}  // namespace pipo
