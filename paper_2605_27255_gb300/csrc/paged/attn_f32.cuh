// Attention of ragged chunks over a paged fp32 cache on the CUDA cores.
//
// out = softmax(scale Q K^T) V for row tiles of 16 RT rows (tokens times the query
// heads of one kv head), a page of 64 entries at a time, everything in fp32; 256
// threads; queries, keys, values and weights pass through shared memory, a thread's
// scores and its part of the output are in registers.  The next page's keys are
// copied under the products with the values, its values under the scores and the
// softmax.  How the threads share a tile depends on its rows (AfGrid, AfRows below).
//
// Measured: six ragged sequences of up to 829 entries with chunks of up to 129 tokens, a window of 256,
// 16 query and 4 kv heads of 64: 36 us, 7.5 TFLOP/s, by latency (a page or two per CTA); one token each
// of 16 sequences of up to 2000 entries, the same heads: 23 us; of two of 2048, 8 heads of 128: 19 us.
//
// The pieces of work and the joining of shared items are those of the bf16
// kernel (work.cuh).
#pragma once

#include <type_traits>

#include "work.cuh"

namespace pipo {

constexpr int kAfThreads = 256;

__host__ __device__ constexpr int af_rows(int rt) { return 16 * rt; }
__host__ __device__ constexpr size_t af_smem(int dh, int rt) {
    // queries and keys (rows padded against bank conflicts), values, weights
    return ((size_t)(af_rows(rt) + kPage) * (dh + 4) + (size_t)kPage * dh + (size_t)af_rows(rt) * (kPage + 4)) * 4;
}
// of a launch: find_pieces uses the same memory before
__host__ __device__ constexpr size_t af_smem_for(int dh, int rt, int batch) {
    return af_smem(dh, rt) > (size_t)find_ints(batch) * 4 ? af_smem(dh, rt) : ((size_t)find_ints(batch) * 4 + 15) / 16 * 16;
}
// CTAs of an SM, by shared memory (dh 64, rt 4: three with 80 registers and a few spilled, 36.6 us for
// the windowed fp32 chunks; two without, 41.5)
__host__ __device__ constexpr int af_ctas(int dh, int rt) {
    return 227 * 1024 / (int)(af_smem(dh, rt) + 2048) < 4 ? 227 * 1024 / (int)(af_smem(dh, rt) + 2048) : 4;
}

// 16 bytes from global to shared memory, or zeros
__device__ __forceinline__ void cp_async16(float* dst, const float* src, bool take) {
    const uint32_t n = take ? 16u : 0u;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
                 "r"(n)
                 : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 64 rows: threads as 16 x 16, thread (ty, tx) has the scores of rows ty + 16 r and entries
// tx + 16 i, and rows ty + 16 r and dims 4 tx + 64 c of the output: 64 multiply-adds per 8 shared
// loads.  Four chunks of 500 tokens up to entry 1000, 16 query and 4 kv heads of 64, 310 us: 20
// TFLOP/s, a quarter of the fp32 rate, with three barriers a page and one buffer each for keys and
// values.  (As in AfRows, with 8 rows per warp: 348 us.)
template <int DH>
struct AfGrid {
    static constexpr int RT = 4, LD = DH + 4, LP = kPage + 4, NC = DH / 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int pos[RT], lo[RT];
    float m[RT], l[RT], o[RT][NC][4];

    template <class F>
    __device__ __forceinline__ void start(F&& range) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            range(ty + 16 * r, pos[r], lo[r]);
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int k = 0; k < NC; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][k][e] = 0.f;
        }
    }
    // scores of a page from entry e0 on, and their weights into p_s
    __device__ __forceinline__ void scores(const float* q_s, const float* k_s, float* p_s, int e0, float c2) {
        float s[RT][4] = {};
#pragma unroll 4
        for (int d = 0; d < DH; d += 4) {
            float4 q[RT], k[4];
#pragma unroll
            for (int r = 0; r < RT; ++r) q[r] = *reinterpret_cast<const float4*>(q_s + (ty + 16 * r) * LD + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = *reinterpret_cast<const float4*>(k_s + (tx + 16 * i) * LD + d);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[r][i] = fmaf(q[r].x, k[i].x, fmaf(q[r].y, k[i].y, fmaf(q[r].z, k[i].z, fmaf(q[r].w, k[i].w, s[r][i]))));
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = m[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = e0 + tx + 16 * i;
                if (e > pos[r] || e < lo[r]) s[r][i] = -INFINITY;
                top = fmaxf(top, s[r][i]);
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            // differences of raw scores, so that the scaling rounds them and not the scores
            const float ref = top == -INFINITY ? 0.f : top, corr = exp2f((m[r] - ref) * c2);
            m[r] = top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = exp2f((s[r][i] - ref) * c2);
                sum += w;
                p_s[(ty + 16 * r) * LP + tx + 16 * i] = w;
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            l[r] = l[r] * corr + sum;
#pragma unroll
            for (int k = 0; k < NC; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][k][e] *= corr;
        }
    }
    __device__ __forceinline__ void values(const float* v_s, const float* p_s) {
#pragma unroll 4
        for (int e = 0; e < kPage; e += 4) {
            float w[RT][4];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(p_s + (ty + 16 * r) * LP + e);
                w[r][0] = x.x; w[r][1] = x.y; w[r][2] = x.z; w[r][3] = x.w;
            }
#pragma unroll
            for (int f = 0; f < 4; ++f)
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    const float4 v = *reinterpret_cast<const float4*>(v_s + (e + f) * DH + 4 * tx + 64 * k);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        o[r][k][0] = fmaf(w[r][f], v.x, o[r][k][0]);
                        o[r][k][1] = fmaf(w[r][f], v.y, o[r][k][1]);
                        o[r][k][2] = fmaf(w[r][f], v.z, o[r][k][2]);
                        o[r][k][3] = fmaf(w[r][f], v.w, o[r][k][3]);
                    }
                }
        }
    }
    // put(row, dim, floats, sum) and stats(row, maximum, sum) of every row, unscaled; every thread of the
    // block comes here
    template <class P, class S>
    __device__ __forceinline__ void finish(P&& put, S&& stats) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = ty + 16 * r;
#pragma unroll
            for (int k = 0; k < NC; ++k) put(row, 4 * tx + 64 * k, o[r][k], l[r]);
            if (tx == 0) stats(row, m[r], l[r]);
        }
    }
};

// 16 rows: two to a warp, a lane has the scores of entries lane and lane + 32 and DH / 32 dims of the
// output.  What a warp shares (queries, weights) is read as a broadcast, and warps without rows
// skip the products.  Bound by the pages' bytes and their latency.  (As in AfGrid, with one row per
// thread: one token each of 16 sequences of up to 2000 entries, 16 query and 4 kv heads of 64, 38 us, so
// 23; of two sequences of 2048, 8 heads of 128, 43 us, so 19.)
template <int DH>
struct AfRows {
    static constexpr int RT = 1, RW = 2, LD = DH + 4, LP = kPage + 4, NC = DH / 32;
    const int lane = threadIdx.x & 31, r0 = (int)(threadIdx.x >> 5) * RW;
    int pos[RW], lo[RW];
    bool live;
    float m[RW], sum[RW], o[RW][NC];

    template <class F>
    __device__ __forceinline__ void start(F&& range) {
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            const bool have = range(r0 + r, pos[r], lo[r]);
            if (r == 0) live = have;
            m[r] = -INFINITY;
            sum[r] = 0.f;
#pragma unroll
            for (int k = 0; k < NC; ++k) o[r][k] = 0.f;
        }
    }
    __device__ __forceinline__ void scores(const float* q_s, const float* k_s, float* p_s, int e0, float c2) {
        if (!live) return;
        float s[RW][2] = {};
#pragma unroll 2
        for (int d = 0; d < DH; d += 4) {
            const float4 k0 = *reinterpret_cast<const float4*>(k_s + lane * LD + d);
            const float4 k1 = *reinterpret_cast<const float4*>(k_s + (lane + 32) * LD + d);
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float4 q = *reinterpret_cast<const float4*>(q_s + (r0 + r) * LD + d);
                s[r][0] = fmaf(q.x, k0.x, fmaf(q.y, k0.y, fmaf(q.z, k0.z, fmaf(q.w, k0.w, s[r][0]))));
                s[r][1] = fmaf(q.x, k1.x, fmaf(q.y, k1.y, fmaf(q.z, k1.z, fmaf(q.w, k1.w, s[r][1]))));
            }
        }
        const int e = e0 + lane;
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            if (e > pos[r] || e < lo[r]) s[r][0] = -INFINITY;
            if (e + 32 > pos[r] || e + 32 < lo[r]) s[r][1] = -INFINITY;
            float top = fmaxf(m[r], fmaxf(s[r][0], s[r][1]));
#pragma unroll
            for (int w = 16; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float ref = top == -INFINITY ? 0.f : top, corr = exp2f((m[r] - ref) * c2);
            m[r] = top;
            const float w0 = exp2f((s[r][0] - ref) * c2), w1 = exp2f((s[r][1] - ref) * c2);
            p_s[(r0 + r) * LP + lane] = w0;
            p_s[(r0 + r) * LP + lane + 32] = w1;
            sum[r] = sum[r] * corr + (w0 + w1);  // this lane's entries; the lanes are added up in finish
#pragma unroll
            for (int k = 0; k < NC; ++k) o[r][k] *= corr;
        }
    }
    __device__ __forceinline__ void values(const float* v_s, const float* p_s) {
        if (!live) return;
#pragma unroll 2
        for (int e = 0; e < kPage; e += 4) {
            float v[4][NC];
#pragma unroll
            for (int f = 0; f < 4; ++f) load_f<float, NC>(v_s + (e + f) * DH + lane * NC, v[f]);
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float4 w = *reinterpret_cast<const float4*>(p_s + (r0 + r) * LP + e);
#pragma unroll
                for (int k = 0; k < NC; ++k)
                    o[r][k] = fmaf(w.x, v[0][k], fmaf(w.y, v[1][k], fmaf(w.z, v[2][k], fmaf(w.w, v[3][k], o[r][k]))));
            }
        }
    }
    template <class P, class S>
    __device__ __forceinline__ void finish(P&& put, S&& stats) {
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            const float L = warp_sum(sum[r]);
            put(r0 + r, lane * NC, o[r], L);
            if (lane == 0) stats(r0 + r, m[r], L);
        }
    }
};

template <int DH, int RT>
__global__ void __launch_bounds__(kAfThreads, af_ctas(DH, RT)) attn_f32_kernel(AttnPagedArgs p, ItemShape shape, int S,
                                                                              int part_rows, size_t part_off) {
    using Tile = std::conditional_t<RT == 1, AfRows<DH>, AfGrid<DH>>;
    static_assert(Tile::RT == RT);
    constexpr int R = af_rows(RT), LD = DH + 4;
    extern __shared__ __align__(16) float af_smem_raw[];
    float* q_s = af_smem_raw;        // [R][LD]
    float* k_s = q_s + R * LD;       // [64][LD]
    float* v_s = k_s + kPage * LD;   // [64][DH]
    float* p_s = v_s + kPage * DH;   // [R][LP]
    __shared__ Piece piece;
    const PagedArgs& c = p.c;
    const int tid = threadIdx.x;
    pdl_launch();
    pdl_wait();
    find_pieces<kAfThreads, 1>(c, shape, (int)blockIdx.x, S, reinterpret_cast<int*>(q_s), &piece);
    if (tid == 0) reinterpret_cast<SharedItem*>(p.scratch)[blockIdx.x] = {0, 0, 0, -1};
    const float c2 = p.scale * 1.4426950408889634f;  // exponents of two
    ItemWalk it;
    it.start(c, shape, piece);
    for (; it.more(); it.next(c, shape)) {
        const int rows = it.tokens(shape) * c.G, i0 = it.tile * shape.TP, np = it.pages(), pg0 = (it.t0 + it.kv0) * 2;
        const int32_t* list =
            shape.n_top > 0 ? p.pages + ((size_t)(it.q0 + it.tile) * c.n_kv + it.g) * shape.n_top : nullptr;
        // entries (in the list's order) that may be read
        int end = it.len;
        if (list) {
            const int pos = it.len - it.n + it.tile, kept = pos < 0 ? 0 : min(shape.n_top, pos / kPage + 1);
            end = kept == 0 ? 0 : (kept - 1) * kPage + (list[kept - 1] == pos / kPage ? pos % kPage + 1 : kPage);
        }
        const int first = first_seen(shape, it.n, it.len, it.tile);
        // page j of this piece into shared memory; what no row sees before the window or past the end becomes zero
        auto copy = [&](float* dst, int ld, const void* pool, int j) {
            const int pg = pg0 + j, dead = first - pg * kPage, live = min(kPage, end - pg * kPage);  // rows [dead, live)
            const bool any = live > max(0, dead);
            const int q = any && list ? list[pg] : pg;
            const float* src = static_cast<const float*>(pool) + (any ? block_off(c, page_block(c, it.b, q), it.g) : 0);
#pragma unroll
            for (int i = 0; i < kPage * DH / 4 / kAfThreads; ++i) {
                const int x = tid + i * kAfThreads, r = x / (DH / 4), d = x % (DH / 4) * 4;
                const bool take = r < live && r >= dead;
                cp_async16(dst + r * ld + d, src + (take ? r * DH + d : 0), take);
            }
            cp_async_commit();
        };
        __syncthreads();  // (find_pieces, or the item before, is done with shared memory)
        for (int x = tid; x < R * (DH / 4); x += kAfThreads) {
            const int r = x / (DH / 4), d = x % (DH / 4) * 4;
            const float* src = static_cast<const float*>(p.q) + (size_t)(it.q0 + i0) * p.ld_q + (size_t)it.g * c.G * DH + d;
            cp_async16(q_s + r * LD + d, r < rows ? src + (size_t)(r / c.G) * p.ld_q + (r % c.G) * DH : src, r < rows);
        }
        copy(k_s, LD, c.k, 0);  // (the queries travel with the first keys)
        copy(v_s, DH, c.v, 0);
        Tile tile;
        // the entries that a row sees (rows past the tile's: those of its last), and whether it is one of the tile's
        tile.start([&](int row, int& pos, int& lo) {
            pos = it.len - it.n + i0 + min(row, rows - 1) / c.G;
            lo = p.window > 0 ? pos - p.window + 1 : 0;
            if (list) pos = end - 1;
            return row < rows;
        });
        for (int j = 0; j < np; ++j) {
            cp_async_wait<1>();  // the keys; the values may be under way
            __syncthreads();
            tile.scores(q_s, k_s, p_s, (pg0 + j) * kPage, c2);
            cp_async_wait<0>();  // the values
            __syncthreads();     // and everyone's weights; the keys are read
            if (j + 1 < np) copy(k_s, LD, c.k, j + 1);
            tile.values(v_s, p_s);
            __syncthreads();
            if (j + 1 < np) copy(v_s, DH, c.v, j + 1);
        }
        const bool whole = it.whole();
        float* part = reinterpret_cast<float*>(p.scratch + part_off) +
                      ((size_t)blockIdx.x * 2 + (it.kv0 == 0 ? 1 : 0)) * part_floats(part_rows, DH);
        tile.finish(
            [&](int row, int d, const auto& o, float l) {
                constexpr int N = (int)(sizeof(o) / sizeof(float));
                if (row >= rows) return;
                const int t = row / c.G;
                const float inv = !whole ? 1.f : l > 0.f ? 1.0f / l : 0.f;
                float* out = static_cast<float*>(p.out) + (size_t)(it.q0 + i0 + t) * p.ld_out + (size_t)(it.g * c.G + row - t * c.G) * DH;
                float x[N];
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = o[e] * inv;
                store_f<float, N>(whole ? out + d : part + ((size_t)(d / 4) * part_rows + row) * 4 + d % 4, x);
            },
            [&](int row, float m, float l) {
                if (!whole && row < rows)
                    *reinterpret_cast<float2*>(part + (size_t)part_rows * DH + 2 * row) = make_float2(m * c2, l);
            });
        if (it.begun() && tid == 0)
            reinterpret_cast<SharedItem*>(p.scratch)[blockIdx.x] = {it.q0 + i0, rows, it.g, it.last_worker(piece)};
    }
}

}  // namespace pipo
