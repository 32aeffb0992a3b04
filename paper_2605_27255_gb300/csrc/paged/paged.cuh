// Device helpers of the paged-cache operators.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "../kernels.cuh"
#include "paged.h"

namespace pipo {

using bf16_t = __nv_bfloat16;

// N consecutive values as fp32 (N * sizeof(T) a multiple of 4 bytes up to 16, aligned to it)
template <typename T, int N>
__device__ __forceinline__ void load_f(const T* p, float (&x)[N]) {
    static_assert(sizeof(T) * N <= 16, "one load");
    struct alignas(sizeof(T) * N) Pack {
        T e[N];
    };
    const Pack v = *reinterpret_cast<const Pack*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f(v.e[i]);
}

template <typename T, int N>
__device__ __forceinline__ void store_f(T* p, const float (&x)[N]) {
    static_assert(sizeof(T) * N <= 16, "one store");
    struct alignas(sizeof(T) * N) Pack {
        T e[N];
    } v;
#pragma unroll
    for (int i = 0; i < N; ++i) v.e[i] = from_f<T>(x[i]);
    *reinterpret_cast<Pack*>(p) = v;
}

// entries of sequence b, its new ones included
__device__ __forceinline__ int seq_len(const PagedArgs& c, int b) {
    return min(max(c.kv_len[b], 0), kPage * c.max_pages);
}

// start of sequence b's rows; clamped, so that no bad offset leaves the token arrays
__device__ __forceinline__ int q_row(const PagedArgs& c, int b) { return min(max(c.q_start[b], 0), c.n_tokens); }

// The block of page p of sequence b; a block outside the pool becomes the
// nearest one inside, so that no read leaves it.
__device__ __forceinline__ int page_block(const PagedArgs& c, int b, int p) {
    return min(max(c.table[(size_t)b * c.max_pages + p], 0), c.n_blocks - 1);
}

// element offset of slot 0 of a block's head g
__device__ __forceinline__ size_t block_off(const PagedArgs& c, int blk, int g) {
    return ((size_t)blk * c.n_kv + g) * kPage * c.dh;
}

// Sequence and position of a new token: b = -1 for a row of no sequence, pos
// < 0 for a token without an entry.
struct Tok {
    int b, pos;
};
__device__ __forceinline__ Tok find_token(const PagedArgs& c, int t) {
    int lo = 0, hi = c.batch;  // the last b with q_start[b] <= t
    while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (q_row(c, m) <= t) lo = m; else hi = m - 1;
    }
    if (lo >= c.batch || q_row(c, lo) > t) return {-1, -1};
    const int end = q_row(c, lo + 1), len = seq_len(c, lo);
    if (t >= end) return {-1, -1};
    return {lo, max(-1, len - (end - t))};
}

// a launch whose blocks may start while the kernel before ends (each waits for it before it reads)
template <typename... P, typename... A>
inline cudaError_t launch_pdl(void (*fn)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, const A&... args) {
    cudaLaunchConfig_t lc{};
    lc.gridDim = grid;
    lc.blockDim = dim3((unsigned)threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, fn, args...);
}

}  // namespace pipo
