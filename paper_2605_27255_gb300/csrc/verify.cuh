// Drafted tokens against the target's probabilities.
//
// Of sequence b's drafts d_1 .. d_n, with target rows p_1 .. p_{n+1} and draft rows q_1 .. q_n (or
// none: q_i is one at d_i): d_i is kept while u_i q_i(d_i) < p_i(d_i).  The last token is
// drawn from max(p_i - q_i, 0) at the first that is not kept, or from p_{n+1}: the first token v
// whose running weight passes floor(r W), W the weight of all.
//
// Weights are probabilities as whole multiples of 2^-44 (63 bits hold 2^19 of
// them), so that sums have no order: any split over threads draws the same token, and the
// rounding, 2^-45 a token, is far below a 32-bit sum's.
//
// A cluster of CTAs per sequence.  Each finds the row by itself (a warp looks at 32 drafts at a time),
// sums its slice of the vocabulary warp by warp, and learns the others' sums through
// distributed shared memory; the one that holds the drawn place goes through the right
// warp's slice once more.  Another CTA's shared memory may be written only once that CTA has started: every
// CTA arrives at the cluster's barrier when it starts and waits there, under the sums, before its first such write.  Bound by the row's read (and the draft row's) and, for few sequences, by
// the chain of start, drafted token, probabilities, row.  Measured back to back with a vocabulary of 151936 in
// fp32: 64 sequences 14.7 us with their 52 MB in L2, 17.9 with rows that are not, one 8.6 us.  Four loads of either row
// in flight take 50 registers, so that 512 CTAs need two rounds (16.8 and 8.0 us in L2); CTAs of 256 threads 17.3 and 12.4.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kernels.cuh"

namespace pipo {

constexpr int kVerThreads = 512, kVerWarps = kVerThreads / 32, kVerCluster = 8;
constexpr int kVerMaxVocab = 1 << 19;  // 2^19 weights of 2^44 at most fit 63 bits

struct VerifyArgs {
    const void *target, *draft;  // [n_drafted + batch][ld_target], [n_drafted][ld_draft] or nullptr
    long long ld_target, ld_draft;
    const int32_t *drafted, *start;  // [n_drafted], [batch + 1]
    const float *u, *r;              // [n_drafted], [batch]
    int vocab, batch, n_drafted, width;
    int32_t *tokens, *count;         // [batch][width], [batch]
};

// N values at p + i, those past n as zeros
template <typename T, int N>
__device__ __forceinline__ void ver_load(const T* p, int i, int n, float (&x)[N]) {
    if (N > 1 && i + N <= n) {
        struct alignas(sizeof(T) * N) Pack {
            T e[N];
        };
        const Pack v = *reinterpret_cast<const Pack*>(p + i);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = to_f(v.e[k]);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = i + k < n ? to_f(p[i + k]) : 0.f;
    }
}

// A probability as a whole multiple of 2^-44 (0 for what is negative or NaN, 1 for what is above), ties to
// even, as hi 2^22 + lo.  Adding 2^23 rounds a number below it to a whole one, whose bits lie
// at the sum's low end; what is left over is exact and is rounded in the same way, at 2^22 times its
// size (conversions to 64-bit integers, a few a cycle of an SM, took half of the kernel's time:
// 30 us for 64 sequences of 151936 tokens).
struct VerWeight {
    int hi, lo;  // 0 .. 2^22, -2^21 .. 2^21
};
__device__ __forceinline__ VerWeight ver_weight(float x) {
    const float a = fminf(fmaxf(x, 0.f), 1.f) * 4194304.f, y = __fadd_rn(a, 8388608.f);
    const float rest = __fsub_rn(a, __fsub_rn(y, 8388608.f)), z = __fmaf_rn(rest, 4194304.f, 12582912.f);
    return {__float_as_int(y) - 0x4b000000, __float_as_int(z) - 0x4b400000};
}
__device__ __forceinline__ unsigned long long ver_sum(int hi, int lo) {
    return (unsigned long long)(((long long)hi << 22) + lo);
}
// a warp's slice has at most 2^19 / 128 tokens, a lane 128 of them: 32 bits hold the sums of either part
static_assert((kVerMaxVocab / (kVerCluster * kVerWarps * 32) + 8LL) * (1 << 22) < (1LL << 31), "a lane's sums");

// floor(r W), 0 <= r < 1: r is m 2^-s with a whole m below 2^24 (s >= 24), m W has 87 bits at most.  (As a product of
// doubles it can end on the next whole number: rows of many ones have a W past 2^53.)
__device__ __forceinline__ unsigned long long ver_place(float r, unsigned long long W) {
    const uint32_t u = __float_as_uint(r), e = max(u >> 23, 1u), m = (u & 0x7fffffu) | (u >> 23 ? 0x800000u : 0u);
    const int s = 150 - (int)e;
    const unsigned long long lo = m * W, hi = __umul64hi(m, W);
    return s < 64 ? lo >> s | hi << (64 - s) : s < 128 ? hi >> (s - 64) : 0ull;
}

template <typename T, int N>
__global__ void __launch_bounds__(kVerThreads) __cluster_dims__(kVerCluster, 1, 1) verify_kernel(VerifyArgs a) {
    namespace cg = cooperative_groups;
    __shared__ int kept_s;
    __shared__ unsigned long long warp_sum[kVerWarps], cta_sum[2][kVerCluster];
    cg::cluster_group cluster = cg::this_cluster();
    const int b = (int)(blockIdx.x / kVerCluster), rank = (int)cluster.block_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // this CTA has started
    pdl_launch();
    pdl_wait();
    const int s0 = min(max(a.start[b], 0), a.n_drafted), s1 = min(max(a.start[b + 1], s0), a.n_drafted);
    const int n = min(s1 - s0, a.width - 1);
    const T* rows = static_cast<const T*>(a.target) + (size_t)(s0 + b) * a.ld_target;
    const T* drafts = static_cast<const T*>(a.draft) + (size_t)s0 * a.ld_draft;
    if (warp == 0) {
        int kept = n;
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            bool ok = true;
            if (i < n) {
                const int t = a.drafted[s0 + i];
                ok = t >= 0 && t < a.vocab;  // (no token: not kept)
                if (ok) {
                    const double q = a.draft ? (double)to_f(drafts[(size_t)i * a.ld_draft + t]) : 1.0;
                    ok = (double)a.u[s0 + i] * q < (double)to_f(rows[(size_t)i * a.ld_target + t]);
                }
            }
            const unsigned no = __ballot_sync(0xffffffffu, !ok);
            if (no) {
                kept = i0 + __ffs(no) - 1;
                break;
            }
        }
        if (lane == 0) kept_s = kept;
    }
    __syncthreads();
    const int kept = kept_s;
    const T* p = rows + (size_t)kept * a.ld_target;
    const bool cut = kept < n;  // a draft was not kept
    const int gone = cut ? a.drafted[s0 + kept] : -1;
    const T* q = cut && a.draft ? drafts + (size_t)kept * a.ld_draft : nullptr;
    int32_t* out = a.tokens + (size_t)b * a.width;
    if (rank == 0) {
        for (int i = threadIdx.x; i < a.width; i += kVerThreads)
            if (i != kept) out[i] = i < kept ? a.drafted[s0 + i] : -1;
        if (threadIdx.x == 0) a.count[b] = kept + 1;
    }
    // this warp's slice, whole vectors
    const int per = (a.vocab + kVerCluster * kVerWarps * N - 1) / (kVerCluster * kVerWarps * N) * N;
    const int i0 = min(a.vocab, (rank * kVerWarps + warp) * per), i1 = min(a.vocab, i0 + per);
    // weights of N tokens from i on; rest: the target's alone (what is left of it has no weight)
    auto weights = [&](int i, bool rest, VerWeight (&w)[N]) {
        float x[N], y[N];
        ver_load<T, N>(p, i, i1, x);
        if (q && !rest) {
            ver_load<T, N>(q, i, i1, y);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = __fsub_rn(x[k], y[k]);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) w[k] = ver_weight(!q && !rest && i + k == gone ? 0.f : x[k]);
    };
    for (int pass = 0; pass < 2; ++pass) {
        int hi = 0, lo = 0;
#pragma unroll 4
        for (int i = i0 + lane * N; i < i1; i += 32 * N) {
            VerWeight w[N];
            weights(i, pass > 0, w);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                hi += w[k].hi;
                lo += w[k].lo;
            }
        }
        unsigned long long mine = ver_sum(hi, lo);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        if (lane == 0) warp_sum[warp] = mine;
        __syncthreads();
        if (pass == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // all have
        if (threadIdx.x < kVerCluster) {
            unsigned long long all = 0;
#pragma unroll
            for (int w = 0; w < kVerWarps; ++w) all += warp_sum[w];
            *cluster.map_shared_rank(&cta_sum[pass][rank], threadIdx.x) = all;
        }
        cluster.sync();
        unsigned long long total = 0, before = 0;
#pragma unroll
        for (int c = 0; c < kVerCluster; ++c) {
            if (c < rank) before += cta_sum[pass][c];
            total += cta_sum[pass][c];
        }
        if (total == 0 && pass == 0) continue;  // (the same for the whole cluster)
        if (total == 0) {
            if (rank == 0 && threadIdx.x == 0) out[kept] = a.vocab - 1;
            return;
        }
        const unsigned long long goal = ver_place(fminf(fmaxf(a.r[b], 0.f), 0.99999994f), total);
        if (goal < before) return;
        for (int w = 0; w < warp; ++w) before += warp_sum[w];
        if (goal < before || goal >= before + warp_sum[warp]) return;
        // the drawn place is in this warp's slice
        for (int i = i0; i < i1; i += 32 * N) {
            VerWeight w[N];
            weights(i + lane * N, pass > 0, w);  // (zeros past the slice's end)
            unsigned long long sum = 0;
#pragma unroll
            for (int k = 0; k < N; ++k) sum += ver_sum(w[k].hi, w[k].lo);
            unsigned long long incl = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, before + incl > goal);
            if (hit) {
                if (lane == __ffs(hit) - 1) {
                    unsigned long long at = before + incl - sum;
                    int v = i + lane * N;
                    for (int k = 0; k < N; ++k) {
                        at += ver_sum(w[k].hi, w[k].lo);
                        if (at > goal) {
                            v += k;
                            break;
                        }
                    }
                    out[kept] = v;
                }
                return;
            }
            before += __shfl_sync(0xffffffffu, incl, 31);
        }
        return;
    }
}

}  // namespace pipo
