// Page scores and the selection of pages.
#pragma once

#include "paged.cuh"

namespace pipo {

// scores[t][g][p] = scale * sum_h q[t, h] . mean[p], all in fp32: the queries of a kv head are
// added up first, then one product per page.  Bound by the means read and the scores written;
// the products are far below the CUDA cores' rate.  Measured (8 kv heads of 128): four tokens over 243
// pages 8 us, 512 tokens over 256 pages 16 us, both by latency.
constexpr int kScorePages = 64;  // pages per CTA

// One token per CTA row (decoding): DH / 16 lanes hold 16 dims each of a page, a warp 512 / DH pages.
// grid (token * n_kv, ceil(max_pages / kScorePages)), 128 threads
template <int DH, typename T>
__global__ void __launch_bounds__(128) page_scores_kernel(ScoreArgs a) {
    constexpr int L = DH / 16, P = 32 / L, V = 16 / sizeof(T);  // lanes per page, pages per warp, values per load
    const PagedArgs& c = a.c;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int t = blockIdx.x / c.n_kv, g = blockIdx.x % c.n_kv, lane = threadIdx.x & 31, d = (lane % L) * 16;
    const Tok k = find_token(c, t);
    if (k.b < 0) return;
    const int seen = k.pos < 0 ? 0 : k.pos / kPage + 1;
    float* o = a.scores + (size_t)blockIdx.x * c.max_pages;
    const int p0 = blockIdx.y * kScorePages, p1 = min(p0 + kScorePages, c.max_pages);
    const int mine = (threadIdx.x >> 5) * P + lane / L;
    float q[16] = {};
    if (p0 < seen)
        for (int h = 0; h < c.G; ++h) {
#pragma unroll
            for (int i = 0; i < 16; i += V) {
                float x[V];
                load_f<T, V>(static_cast<const T*>(a.q) + (size_t)t * a.ld_q + (size_t)(g * c.G + h) * DH + d + i, x);
#pragma unroll
                for (int e = 0; e < V; ++e) q[i + e] += x[e];
            }
        }
#pragma unroll
    for (int r = 0; r < kScorePages / (4 * P); ++r) {
        const int p = p0 + r * 4 * P + mine;
        float s = 0.f;
        if (p < seen) {
            const T* m = static_cast<const T*>(c.means) + ((size_t)page_block(c, k.b, p) * c.n_kv + g) * DH + d;
#pragma unroll
            for (int i = 0; i < 16; i += V) {
                float x[V];
                load_f<T, V>(m + i, x);
#pragma unroll
                for (int e = 0; e < V; ++e) s = fmaf(q[i + e], x[e], s);
            }
        }
#pragma unroll
        for (int w = L / 2; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
        if (lane % L == 0 && p < p1) o[p] = p < seen ? s * a.scale : -INFINITY;
    }
}

// Chunks: kScoreTok tokens of one sequence and 64 pages per CTA, products in register tiles of 2
// tokens x 4 pages, both operands in shared memory as fp32 (rows padded against bank conflicts).
// grid (row tiles * n_kv, ceil(max_pages / kScorePages)), 256 threads.  One warp per token and page
// range, as above, read every mean again for every token (84 us for 512 tokens and 256 pages).
constexpr int kScoreTok = 32;
__host__ __device__ constexpr size_t score_smem(int dh) { return (size_t)(kScoreTok + kScorePages) * (dh + 4) * 4; }

template <int DH, typename T>
__global__ void __launch_bounds__(256) page_scores_chunk_kernel(ScoreArgs a) {
    constexpr int LD = DH + 4, V = 16 / sizeof(T), C = DH / V;
    extern __shared__ __align__(16) float sc_smem[];
    float* qs = sc_smem;                   // [kScoreTok][LD]
    float* ms = sc_smem + kScoreTok * LD;  // [kScorePages][LD]
    const PagedArgs& c = a.c;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int g = blockIdx.x % c.n_kv, lane = threadIdx.x & 31;
    // the row tile's sequence (every warp finds it for itself)
    int r = blockIdx.x / c.n_kv, b = -1, tile = 0;
    for (int b0 = 0; b0 < c.batch; b0 += 32) {
        const int n = b0 + lane < c.batch ? (max(0, q_row(c, b0 + lane + 1) - q_row(c, b0 + lane)) + kScoreTok - 1) / kScoreTok : 0;
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
            tile = __shfl_sync(0xffffffffu, r - (incl - n), src);
            break;
        }
        r -= __shfl_sync(0xffffffffu, incl, 31);
    }
    if (b < 0) return;
    const int t0 = q_row(c, b) + tile * kScoreTok, end = q_row(c, b + 1), nt = min(kScoreTok, end - t0);
    const int len = seq_len(c, b), pos0 = len - (end - t0);  // position of the first token
    const int p0 = blockIdx.y * kScorePages, p1 = min(p0 + kScorePages, c.max_pages);
    const int last = pos0 + nt - 1, seen = last < 0 ? 0 : last / kPage + 1;  // pages that any of the tokens sees
    if (p0 < seen) {
        for (int i = threadIdx.x; i < kScoreTok * C; i += 256) {
            const int t = i / C, d = (i % C) * V;
            float x[V] = {};
            if (t < nt)
                for (int h = 0; h < c.G; ++h) {
                    float y[V];
                    load_f<T, V>(static_cast<const T*>(a.q) + (size_t)(t0 + t) * a.ld_q + (size_t)(g * c.G + h) * DH + d, y);
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] += y[e];
                }
#pragma unroll
            for (int e = 0; e < V; e += 4)
                *reinterpret_cast<float4*>(qs + t * LD + d + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        }
#pragma unroll 4
        for (int i = threadIdx.x; i < kScorePages * C; i += 256) {
            const int p = i / C, d = (i % C) * V;
            float x[V] = {};
            if (p0 + p < seen)
                load_f<T, V>(static_cast<const T*>(c.means) + ((size_t)page_block(c, b, p0 + p) * c.n_kv + g) * DH + d, x);
#pragma unroll
            for (int e = 0; e < V; e += 4)
                *reinterpret_cast<float4*>(ms + p * LD + d + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        }
        __syncthreads();
    }
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;  // pages tx + 16 i, tokens ty + 16 j
    float acc[2][4] = {};
    if (p0 < seen) {
#pragma unroll 4
        for (int d = 0; d < DH; d += 4) {
            float4 q[2], m[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) q[j] = *reinterpret_cast<const float4*>(qs + (ty + 16 * j) * LD + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = *reinterpret_cast<const float4*>(ms + (tx + 16 * i) * LD + d);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[j][i] = fmaf(q[j].x, m[i].x, fmaf(q[j].y, m[i].y, fmaf(q[j].z, m[i].z, fmaf(q[j].w, m[i].w, acc[j][i]))));
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int t = ty + 16 * j, pos = pos0 + t;
        if (t >= nt) continue;
        const int sees = pos < 0 ? 0 : pos / kPage + 1;
        float* o = a.scores + ((size_t)(t0 + t) * c.n_kv + g) * c.max_pages;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = p0 + tx + 16 * i;
            if (p < p1) o[p] = p < sees ? acc[j][i] * a.scale : -INFINITY;
        }
    }
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
// KPL > 0: a lane holds the keys of pages l, l + 32, ... in KPL registers (at most 32 KPL pages);
// read from memory for each of the 32 bits they took 19 us for 243 pages.  KPL = 0: any number.
template <int KPL>
__global__ void __launch_bounds__(128) page_select_kernel(SelectArgs a) {
    const PagedArgs& c = a.c;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int l = threadIdx.x & 31;
    if (w >= (long long)c.n_tokens * c.n_kv) return;
    const Tok k = find_token(c, (int)(w / c.n_kv));
    if (k.b < 0) return;
    int32_t* o = a.pages + (size_t)w * a.n_top;
    const float* sc = a.scores + (size_t)w * c.max_pages;
    uint32_t* bits = a.bits ? a.bits + (size_t)w * bit_words(c.max_pages) : nullptr;
    const int seen = k.pos < 0 ? 0 : k.pos / kPage + 1;
    const int head = min(a.n_sink, seen), tail = max(head, seen - a.n_local);  // candidates: [head, tail)
    const int want = min(a.n_top, seen) - (seen - tail + head);                 // of them to be kept
    constexpr int NK = KPL > 0 ? KPL : 1;
    uint32_t keys[NK];
    if (KPL > 0) {
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int p = 32 * i + l;
            keys[i] = p >= head && p < tail ? score_key(sc[p]) : 0u;
        }
    }
    // candidates with a key of at least x (x > 0)
    auto reach = [&](uint32_t x) {
        int n = 0;
        if (KPL > 0) {
#pragma unroll
            for (int i = 0; i < NK; ++i) n += keys[i] >= x;
        } else {
            for (int p = head + l; p < tail; p += 32) n += score_key(sc[p]) >= x;
        }
        return (int)__reduce_add_sync(0xffffffffu, n);
    };
    uint32_t key = 0;  // the smallest key that is kept
    int ties = want;   // and how many of it: all, where every candidate is kept
    if (want < tail - head && want > 0) {
        for (int bit = 31; bit >= 0; --bit)
            if (reach(key | (1u << bit)) >= want) key |= 1u << bit;
        ties = want - (key == 0xffffffffu ? 0 : reach(key + 1));
    } else if (want <= 0) {
        key = 0xffffffffu;  // none (a NaN of this key does not exist)
        ties = 0;
    } else {
        ties = tail - head;
    }
    int n = 0;
    auto emit = [&](int p, uint32_t x) {  // 32 pages in order
        const bool cand = p >= head && p < tail;
        const unsigned eq = __ballot_sync(0xffffffffu, cand && x == key);
        const bool keep = p < seen && (!cand || x > key || (x == key && __popc(eq & ((1u << l) - 1u)) < ties));
        const unsigned kept = __ballot_sync(0xffffffffu, keep);
        if (keep) o[n + __popc(kept & ((1u << l) - 1u))] = p;
        n += __popc(kept);
        ties -= min(ties, (int)__popc(eq));
        if (bits && l == 0) bits[p / 32] = kept;
    };
    if (KPL > 0) {
#pragma unroll
        for (int i = 0; i < NK; ++i)
            if (32 * i < seen) emit(32 * i + l, keys[i]);
    } else {
        for (int p0 = 0; p0 < seen; p0 += 32) {
            const int p = p0 + l;
            emit(p, p >= head && p < tail ? score_key(sc[p]) : 0u);
        }
    }
    for (int i = n + l; i < a.n_top; i += 32) o[i] = -1;
    if (bits)
        for (int i = (seen + 31) / 32 + l; i < bit_words(c.max_pages); i += 32) bits[i] = 0u;
}

}  // namespace pipo
