// Attention of ragged chunks over a paged fp32 cache on the CUDA cores.
//
// out = softmax(scale Q K^T) V for row tiles of 16 RT rows (tokens times the query
// heads of one kv head), a page of 64 entries at a time, everything in fp32:
// 256 threads as 16 x 16, thread (ty, tx) has the scores of rows ty + 16 r and
// entries tx + 16 i, and rows ty + 16 r and dims 4 tx + 64 c of the output, both in
// registers; queries, keys, values and weights pass through shared memory.  The next
// page's keys are copied under the products with the values, its values under
// the scores and the softmax.  Bound by the fp32 rate (RT = 4: 64 multiply-adds per 8
// shared loads) or, with few rows (RT = 1), by the pages' bytes.
//
// Measured: six ragged sequences of up to 829 entries with chunks of up to 129 tokens, a window of 256,
// 16 query and 4 kv heads of 64: 36 us, 7.5 TFLOP/s, by latency (a page or two per CTA); one token of
// 52 entries 8 us.
//
// The pieces of work and the joining of shared items are those of the bf16
// kernel (work.cuh).
#pragma once

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

template <int DH, int RT>
__global__ void __launch_bounds__(kAfThreads, af_ctas(DH, RT)) attn_f32_kernel(AttnPagedArgs p, ItemShape shape, int S,
                                                                              int part_rows, size_t part_off) {
    constexpr int R = af_rows(RT), LD = DH + 4, LP = kPage + 4, NC = DH / 64;
    extern __shared__ __align__(16) float af_smem_raw[];
    float* q_s = af_smem_raw;        // [R][LD]
    float* k_s = q_s + R * LD;       // [64][LD]
    float* v_s = k_s + kPage * LD;   // [64][DH]
    float* p_s = v_s + kPage * DH;   // [R][LP]
    __shared__ Piece piece;
    const PagedArgs& c = p.c;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
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
        // page j of this piece into shared memory; what lies past the end becomes zero
        auto copy = [&](float* dst, int ld, const void* pool, int j) {
            const int pg = pg0 + j, live = min(kPage, end - pg * kPage);
            const int q = live > 0 ? (list ? list[pg] : pg) : 0;
            const float* src = static_cast<const float*>(pool) + (live > 0 ? block_off(c, page_block(c, it.b, q), it.g) : 0);
#pragma unroll
            for (int i = 0; i < kPage * DH / 4 / kAfThreads; ++i) {
                const int x = tid + i * kAfThreads, r = x / (DH / 4), d = x % (DH / 4) * 4;
                cp_async16(dst + r * ld + d, src + (r < live ? r * DH + d : 0), r < live);
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
        int pos[RT], lo[RT];
        float m[RT], l[RT], o[RT][NC][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            pos[r] = it.len - it.n + i0 + min(ty + 16 * r, rows - 1) / c.G;
            lo[r] = p.window > 0 ? pos[r] - p.window + 1 : 0;
            if (list) pos[r] = end - 1;
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int k = 0; k < NC; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][k][e] = 0.f;
        }
        for (int j = 0; j < np; ++j) {
            cp_async_wait<1>();  // the keys; the values may be under way
            __syncthreads();
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
            const int e0 = (pg0 + j) * kPage;
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
            cp_async_wait<0>();  // the values
            __syncthreads();     // and everyone's weights; the keys are read
            if (j + 1 < np) copy(k_s, LD, c.k, j + 1);
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
            __syncthreads();
            if (j + 1 < np) copy(v_s, DH, c.v, j + 1);
        }
        const bool whole = it.whole();
        float* part = reinterpret_cast<float*>(p.scratch + part_off) +
                      ((size_t)blockIdx.x * 2 + (it.kv0 == 0 ? 1 : 0)) * part_floats(part_rows, DH);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = ty + 16 * r, t = row / c.G;
            if (row >= rows) continue;
            const float inv = !whole ? 1.f : l[r] > 0.f ? 1.0f / l[r] : 0.f;
            float* out = static_cast<float*>(p.out) + (size_t)(it.q0 + i0 + t) * p.ld_out + (size_t)(it.g * c.G + row - t * c.G) * DH;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = o[r][k][e] * inv;
                store_f<float, 4>(whole ? out + 4 * tx + 64 * k : part + ((size_t)(tx + 16 * k) * part_rows + row) * 4, x);
            }
            if (!whole && tx == 0)
                *reinterpret_cast<float2*>(part + (size_t)part_rows * DH + 2 * row) = make_float2(m[r] * c2, l[r]);
        }
        if (it.begun() && tid == 0)
            reinterpret_cast<SharedItem*>(p.scratch)[blockIdx.x] = {it.q0 + i0, rows, it.g, it.last_worker(piece)};
    }
}

}  // namespace pipo
