// Attention of few rows per sequence over a paged cache of e4m3 codes.
//
// out = softmax(scale q . (s_k c_k)) (s_v c_v) for row tiles of 8 NT rows (tokens times the
// query heads of one kv head).  With few rows the cache's bytes are the time, so codes go from
// the copies' shared memory to registers once and become MMA operands there (mma.sync, fp16
// with fp32 sums: an e4m3 code is an fp16 number), without a detour through an fp16
// tile.  Entries and dims are the MMAs' rows, so that the few queries fill its 8 columns:
//   S^T = C_k Q^T   16 entries x 8 rows, a step of 16 dims each; which dims a step takes is
//                   free as long as both sides agree, so a lane reads 16 bytes of an entry
//                   at a time;
//   O^T += C_v^T P^T  16 dims x 8 rows; a lane reads 16 dims of four entries and pairs the
//                   entries' bytes.  P^T comes from S^T's registers by movmatrix.
// The queries are scaled by a power of two per row to fp16, the largest below 2^15 (bf16's digits fit down to 2^-31 of
// it, what is below 2^-39 is lost), scores get it back with the block's scale in fp32.  The values'
// scales go into the weights (codes.cuh), which keep fp16's 11 digits.
//
// A warp takes 16 (or 32) entries of a 128-entry unit, with its own ring of copies, running maximum
// and output; warps meet only at the end of an item, where their outputs are joined in
// order.  Nothing waits on anything but its own copies.
//
// The pieces of work and the joining of shared items are those of work.cuh.
//
// Bound by HBM while it streams, else by its start (lengths, piece, block table, one after the other: 5 us) and the
// joining.  Measured with the joining, back to back: eight sequences of 15.5 K entries with one token each, 32 query
// and 8 kv heads of 128, 47 us, 5.4 TB/s (49 with two such caches in turn); 64 sequences of five tokens with a window of
// 1024, 16 heads of 64, 32 to 39 us (by the GPU), 3.5 to 4.2 TB/s; one token over 1155 entries 9.0 us.
#pragma once

#include <cuda_fp16.h>

#include "codes.cuh"
#include "work.cuh"

namespace pipo {

// Entries of a warp's step: 16 fill an MMA's rows, 32 share a step's other work (eight sequences of 15.5 K
// entries 49.1 -> 47.7 us); with more than one column tile their scores would not fit the registers.
__host__ __device__ constexpr int few_entries(int, int nt) { return nt == 1 ? 32 : 16; }
__host__ __device__ constexpr int few_warps(int dh, int nt) { return kTileEnt / few_entries(dh, nt); }
__host__ __device__ constexpr int few_threads(int dh, int nt) { return 32 * few_warps(dh, nt); }
__host__ __device__ constexpr int few_ctas(int dh, int nt) { return nt > 2 ? 1 : dh == 64 && nt == 1 ? 4 : 2; }  // of an SM
__host__ __device__ constexpr int few_stages(int dh, int nt) { return nt > 2 ? 4 : nt == 1 && dh == 128 ? 3 : 2; }
__host__ __device__ constexpr int few_stage_bytes(int dh, int nt) { return 2 * few_entries(dh, nt) * dh; }  // a step's keys and values
__host__ __device__ constexpr int few_ring_bytes(int dh, int nt) {
    return few_warps(dh, nt) * few_stages(dh, nt) * few_stage_bytes(dh, nt);
}
__host__ __device__ constexpr int few_q_bytes(int dh, int nt) { return nt > 1 ? nt * 8 * dh * 2 : 0; }
// four warps' outputs and their (maximum, sum); the 16-byte chunks of a row are swizzled by it
__host__ __device__ constexpr int few_join_bytes(int dh, int nt) { return 4 * nt * 8 * (dh + 2) * 4; }
template <int DH>
__device__ __forceinline__ int few_join_at(int r, int chunk) { return r * DH + ((chunk ^ ((r >> 1) & 3)) << 2); }
__host__ __device__ constexpr size_t few_smem(int dh, int nt, int batch) {
    const size_t n = (size_t)few_ring_bytes(dh, nt) + few_join_bytes(dh, nt) + few_q_bytes(dh, nt);
    const size_t find = ((size_t)find_ints(batch) * 4 + 15) / 16 * 16;
    return n > find ? n : find;
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turn8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// 16 bytes (or the first n of them, then zeros) into shared memory
__device__ __forceinline__ void copy16(uint32_t to, const void* from, uint32_t n) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(n) : "memory");
}
__device__ __forceinline__ bool few_large(float m) { return fabsf(m) > kLargeScore && m > kNoScore; }
// byte offsets of 16-byte chunk c of entry r (0 .. 15) in a stage's keys or values: swizzled so that the
// lanes' reads hit different banks (keys: lanes take neighbouring entries; values: every other one)
template <int DH>
__device__ __forceinline__ uint32_t few_k_off(int r, int c) {
    return DH == 128 ? (uint32_t)(r * 128 + ((c ^ ((r & 1) << 2)) << 4)) : (uint32_t)(r * 64 + (c << 4));
}
template <int DH>
__device__ __forceinline__ uint32_t few_v_off(int r, int c) {
    return DH == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 6)) << 4)) : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}

template <int DH, int NT>
__global__ void __launch_bounds__(few_threads(DH, NT), few_ctas(DH, NT)) attn_few8_kernel(AttnPagedArgs p, ItemShape shape, int S,
                                                                             int part_rows, size_t part_off) {
    constexpr int EW = few_entries(DH, NT), WARPS = few_warps(DH, NT), THREADS = 32 * WARPS, ET = EW / 16;
    constexpr int ST = few_stages(DH, NT), SB = few_stage_bytes(DH, NT), KS = DH / 16, MT = DH / 16, ROWS = 8 * NT;
    constexpr int NC = EW * DH / 16 / 32;  // 16-byte chunks of a lane, of a stage's keys or values
    constexpr int VS = EW * DH;            // the values' place in a stage
    extern __shared__ __align__(128) unsigned char few_raw[];
    __shared__ Piece piece[1];
    __shared__ float row_scale[NT > 1 ? ROWS : 1];
    __shared__ float scales[WARPS][ST][2];  // of the block that a stage holds: keys', values'
    unsigned char* ring = few_raw;
    float* join_s = reinterpret_cast<float*>(few_raw + few_ring_bytes(DH, NT));
    // queries in the order of the MMAs' registers (with one column tile every warp has them in registers)
    uint2* q_s = reinterpret_cast<uint2*>(few_raw + few_ring_bytes(DH, NT) + few_join_bytes(DH, NT));
    const PagedArgs& c = p.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane >> 2, tig = lane & 3;
    const int me = (int)blockIdx.x;
    pdl_wait();
    find_pieces<THREADS, 1>(c, shape, me, S, reinterpret_cast<int*>(few_raw), piece);
    pdl_launch();
    if (threadIdx.x == 0) reinterpret_cast<SharedItem*>(p.scratch)[me] = {0, 0, 0, -1};
    __syncthreads();

    const float c2 = p.scale * 1.4426950408889634f;  // exponents of two
    unsigned char* mine_s = ring + (size_t)warp * ST * SB;

    // ---- copies: this warp's entries of unit lu of item ld.  They lie side by side, 16 bytes of a lane 512 apart,
    // in the cache and (swizzled within) in the stage.
    constexpr int RS = 512 / DH;  // entries between a lane's chunks
    const int r0 = lane / (DH / 16), ch = lane % (DH / 16);
    const uint32_t stage_at = (uint32_t)__cvta_generic_to_shared(mine_s), k_to = stage_at + few_k_off<DH>(r0, ch);
    const uint32_t v_to[2] = {stage_at + VS + few_v_off<DH>(r0, ch), stage_at + VS + few_v_off<DH>(RS + r0, ch) - 512};
    const uint32_t scale_to = (uint32_t)__cvta_generic_to_shared(&scales[warp][0][lane & 1]);
    const float* scale_from = lane ? p.v_scale : p.k_scale;
    ItemWalk ld;
    ld.start(c, shape, piece[0]);
    int lu = ld.kv0, held = lu - 32, blocks = -1, slot_in = 0;  // lane l has the block of unit held + l
    auto issue = [&]() {
        if (ld.more()) {
            const int first = first_seen(shape, ld.n, ld.len, ld.tile);
            if (lu >= held + 32) {
                held = lu;
                const int page = (ld.t0 + lu + lane) * 2 + warp * EW / kPage;
                blocks = lu + lane < ld.kv1 && (long long)page * kPage < ld.len && page >= first / kPage
                             ? page_block(c, ld.b, page)
                             : -1;
            }
            const int blk = __shfl_sync(0xffffffffu, blocks, lu - held);
            const int e0 = (ld.t0 + lu) * kTileEnt + warp * EW;
            const size_t head = (size_t)max(blk, 0) * c.n_kv + ld.g, off = (head * kPage + warp * EW % kPage) * DH + lane * 16;
            const uint8_t *k = static_cast<const uint8_t*>(c.k) + off, *v = static_cast<const uint8_t*>(c.v) + off;
            const uint32_t to = slot_in * SB;
            if (blk >= 0 && e0 >= first && e0 + EW <= ld.len) {
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    copy16(k_to + to + i * 512, k + i * 512, 16u);
                    copy16(v_to[i & 1] + to + i * 512, v + i * 512, 16u);
                }
            } else {
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const int e = e0 + r0 + i * RS;
                    const uint32_t nb = blk >= 0 && e >= first && e < ld.len ? 16u : 0u;
                    copy16(k_to + to + i * 512, k + i * 512, nb);
                    copy16(v_to[i & 1] + to + i * 512, v + i * 512, nb);
                }
            }
            if (lane < 2)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(scale_to + slot_in * 8), "l"(scale_from + head),
                             "r"(blk >= 0 ? 4u : 0u)
                             : "memory");
            if (++lu == ld.kv1) {
                ld.next(c, shape);
                lu = ld.kv0;
                held = lu - 32;
            }
        }
        cp_async_commit();
        slot_in = slot_in + 1 == ST ? 0 : slot_in + 1;
    };
#pragma unroll 1
    for (int i = 0; i < ST - 1; ++i) issue();

    ItemWalk it;
    it.start(c, shape, piece[0]);
    int slot = 0;
    // (one column tile) an item's queries: a lane has row grp, 16 dims from 16 tig (and 64 + 16 tig) on, as its keys
    uint4 x[NT == 1 ? DH / 64 : 1][2];
    auto load_queries = [&]() {
        if (NT > 1 || !it.more()) return;
        const bool live = grp < it.tokens(shape) * c.G;
        const int t = live ? grp / c.G : 0;
        const bf16_t* q = static_cast<const bf16_t*>(p.q) + (size_t)(it.q0 + it.tile * shape.TP + t) * p.ld_q +
                          (size_t)(it.g * c.G + (live ? grp - t * c.G : 0)) * DH + tig * 16;
#pragma unroll
        for (int h = 0; h < DH / 64; ++h)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                x[NT == 1 ? h : 0][k] = live ? *reinterpret_cast<const uint4*>(q + h * 64 + k * 8) : make_uint4(0u, 0u, 0u, 0u);
    };
    load_queries();
    while (it.more()) {
        const int rows = it.tokens(shape) * c.G, i0 = it.tile * shape.TP;
        // ---- queries
        uint2 qf[NT == 1 ? KS : 1];
        float scale_of_row[2] = {1.f, 1.f};  // (one column tile) of this lane's rows 2 tig, 2 tig + 1
        if constexpr (NT == 1) {
            // every warp for itself, loaded before the item that went before was joined
            float most = 0.f;
#pragma unroll
            for (int h = 0; h < DH / 64; ++h)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t u[4] = {x[NT == 1 ? h : 0][k].x, x[NT == 1 ? h : 0][k].y, x[NT == 1 ? h : 0][k].z, x[NT == 1 ? h : 0][k].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(finite_abs(bf_lo(u[e])), finite_abs(bf_hi(u[e]))));
                }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int ex = query_exponent(most);
            const float sc = exp2_int(ex), f = exp2_int(-ex);
            scale_of_row[0] = __shfl_sync(0xffffffffu, sc, 8 * tig);
            scale_of_row[1] = __shfl_sync(0xffffffffu, sc, 8 * tig + 4);
#pragma unroll
            for (int h = 0; h < DH / 64; ++h)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    qf[NT == 1 ? h * 4 + 2 * k : 0] = make_uint2(half2_of(bf_lo(x[NT == 1 ? h : 0][k].x) * f, bf_hi(x[NT == 1 ? h : 0][k].x) * f),
                                                                half2_of(bf_lo(x[NT == 1 ? h : 0][k].y) * f, bf_hi(x[NT == 1 ? h : 0][k].y) * f));
                    qf[NT == 1 ? h * 4 + 2 * k + 1 : 0] = make_uint2(half2_of(bf_lo(x[NT == 1 ? h : 0][k].z) * f, bf_hi(x[NT == 1 ? h : 0][k].z) * f),
                                                                    half2_of(bf_lo(x[NT == 1 ? h : 0][k].w) * f, bf_hi(x[NT == 1 ? h : 0][k].w) * f));
                }
        } else {
            // a warp per row, four dims a lane
            for (int r = warp; r < ROWS; r += WARPS) {
                float x[4] = {0.f, 0.f, 0.f, 0.f}, most = 0.f;
                if (r < rows && lane < DH / 4) {
                    const int t = r / c.G;
                    load_f<bf16_t, 4>(static_cast<const bf16_t*>(p.q) + (size_t)(it.q0 + i0 + t) * p.ld_q +
                                          (size_t)(it.g * c.G + r - t * c.G) * DH + lane * 4,
                                      x);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, finite_abs(x[i]));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                const int ex = query_exponent(most);
                const float f = exp2_int(-ex);
                if (lane == 0) row_scale[r] = exp2_int(ex);
                if (lane < DH / 4) {  // dims 4 lane ..: chunk lane / 4, word lane % 4 of it
                    const int step = (lane >> 4) * 4 + (lane & 3), quad = (lane >> 2) & 3;
                    q_s[((r >> 3) * KS + step) * 32 + (r & 7) * 4 + quad] = make_uint2(half2_of(x[0] * f, x[1] * f), half2_of(x[2] * f, x[3] * f));
                }
            }
            __syncthreads();
        }
        // ---- this lane's rows: 2 tig and 2 tig + 1 of every column tile
        float cs[NT][2], m[NT][2], l[NT][2], v_ref[NT][2], o[NT][MT][4];  // (references m + v_ref: codes.cuh)
        int pos[NT][2], lo[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = min(t * 8 + 2 * tig + h, rows - 1);
                cs[t][h] = c2 * (NT == 1 ? scale_of_row[h] : row_scale[NT > 1 ? t * 8 + 2 * tig + h : 0]);
                pos[t][h] = it.len - it.n + i0 + r / c.G;
                lo[t][h] = p.window > 0 ? pos[t][h] - p.window + 1 : 0;
                m[t][h] = kNoScore;
                v_ref[t][h] = 0.f;
                l[t][h] = 0.f;
            }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][i][e] = 0.f;
        // entries that every row sees: all before `free_to`, from `free_from` on
        const int free_to = it.len - it.n + i0 + 1;
        const int free_from = p.window > 0 ? it.len - it.n + i0 + it.tokens(shape) - p.window : 0;
        bool large = false;      // (the same for the warp) large scores among its rows' references
        float v_top = kNoScale;  // the largest scale so far
        for (int u = it.kv0; u < it.kv1; ++u) {
            cp_async_wait<ST - 2>();
            __syncwarp();
            issue();
            const unsigned char* ks_s = mine_s + slot * SB;
            const unsigned char* vs_s = ks_s + VS;
            const float k_scale = scales[warp][slot][0], v_now = log2_scale(scales[warp][slot][1]);
            slot = slot + 1 == ST ? 0 : slot + 1;
            const int e0 = (it.t0 + u) * kTileEnt + warp * EW;
            // (the sums of the two halves of the dims apart where registers allow: shorter chains)
            constexpr int CH = DH == 128 && NT == 1 ? 2 : 1;
            float s[ET][NT][4], s2[CH][ET][NT][4];
#pragma unroll
            for (int x = 0; x < ET; ++x)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int h = 0; h < CH; ++h) s2[h][x][t][e] = 0.f;
            uint4 kw[ET][2][DH / 64];
#pragma unroll
            for (int x = 0; x < ET; ++x)
#pragma unroll
                for (int half = 0; half < DH / 64; ++half) {
                    kw[x][0][half] = *reinterpret_cast<const uint4*>(ks_s + few_k_off<DH>(16 * x + grp, tig + 4 * half));
                    kw[x][1][half] = *reinterpret_cast<const uint4*>(ks_s + few_k_off<DH>(16 * x + grp + 8, tig + 4 * half));
                }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int half = 0; half < DH / 64; ++half)
#pragma unroll
                    for (int x = 0; x < ET; ++x) {
                        const uint4 ka = kw[x][0][half], kb = kw[x][1][half];
                        const uint32_t a = i == 0 ? ka.x : i == 1 ? ka.y : i == 2 ? ka.z : ka.w;
                        const uint32_t b = i == 0 ? kb.x : i == 1 ? kb.y : i == 2 ? kb.z : kb.w;
                        const uint32_t a0 = decode_lo(a), a1 = decode_lo(b), a2 = decode_hi(a), a3 = decode_hi(b);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            const uint2 q = NT == 1 ? qf[NT == 1 ? half * 4 + i : 0] : q_s[(t * KS + half * 4 + i) * 32 + lane];
                            mma_f16(s2[half % CH][x][t], a0, a1, a2, a3, q.x, q.y);
                        }
                    }
            // ---- softmax: s[.][t][0], s[.][t][1] are entry grp's scores for the lane's two rows, [2], [3] entry
            // grp + 8's, in the raw (times f).  The references of the exponents move when a score (with its scale) has passed
            // one by 2^8 (as in the tile kernel); only then the warp agrees on its maxima.
            const bool edge = e0 + EW > free_to || e0 < free_from;
            const float v_up = v_now + kWeightUp;
            const bool far = v_now < v_top - kFarScale;  // (the same for the warp)
            bool move = large || far;
            float down = code_ex2(-v_up);  // from weights to the sum's
            v_top = fmaxf(v_top, v_now);
            float top[NT][2], f[NT][2], neg[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    f[t][h] = fmaxf(cs[t][h] * k_scale, 1.17549435e-38f);  // (never 0: masked scores are -infinity)
                    neg[t][h] = v_up - (m[t][h] + v_ref[t][h]);
                    top[t][h] = -INFINITY;
#pragma unroll
                    for (int x = 0; x < ET; ++x) {
#pragma unroll
                        for (int e = h; e < 4; e += 2) s[x][t][e] = CH == 2 ? s2[0][x][t][e] + s2[CH - 1][x][t][e] : s2[0][x][t][e];
                        if (edge) {
                            const int a = e0 + 16 * x + grp;
                            if (a > pos[t][h] || a < lo[t][h]) s[x][t][h] = -INFINITY;
                            if (a + 8 > pos[t][h] || a + 8 < lo[t][h]) s[x][t][2 + h] = -INFINITY;
                        }
                        top[t][h] = fmaxf(top[t][h], fmaxf(s[x][t][h], s[x][t][2 + h]));
                    }
                    top[t][h] *= f[t][h];
                    move |= top[t][h] + neg[t][h] > kWeightTop;
                }
            if (__any_sync(0xffffffffu, move)) {
                bool big = false;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) top[t][h] = fmaxf(top[t][h], __shfl_xor_sync(0xffffffffu, top[t][h], w));
                        const float by = (m[t][h] - top[t][h]) + (v_ref[t][h] - v_now);
                        if (by < 0.f) {
                            m[t][h] = top[t][h];
                            v_ref[t][h] = v_now;
                            l[t][h] = times_ex2(l[t][h], by);
                            const float y = code_ex2(by);
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                o[t][i][h] *= y;
                                o[t][i][2 + h] *= y;
                            }
                        }
                        neg[t][h] = v_up - (m[t][h] + v_ref[t][h]);
                        big |= few_large(m[t][h]);
                    }
                large = __any_sync(0xffffffffu, big);
                if (large) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int x = 0; x < ET; ++x)
#pragma unroll
                                for (int e = h; e < 4; e += 2) s[x][t][e] = __fsub_rn(__fmul_rn(s[x][t][e], f[t][h]), m[t][h]);
                            f[t][h] = 1.f;
                            neg[t][h] = v_up - v_ref[t][h];
                        }
                }
                if (far) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int x = 0; x < ET; ++x)
#pragma unroll
                                for (int e = h; e < 4; e += 2) l[t][h] += code_ex2(fmaf(s[x][t][e], f[t][h], neg[t][h] - v_up));
                    down = 0.f;
                }
            }
            uint32_t pb[ET][NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int x = 0; x < ET; ++x) {
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = code_ex2(fmaf(s[x][t][e], f[t][e & 1], neg[t][e & 1]));
#pragma unroll
                    for (int h = 0; h < 2; ++h) sum[h] += w[h] + w[2 + h];
                    pb[x][t][0] = turn8x8(half2_of(w[0], w[1]));
                    pb[x][t][1] = turn8x8(half2_of(w[2], w[3]));
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) l[t][h] = fmaf(sum[h], down, l[t][h]);
            }
            // ---- values: dims 16 grp .. (8 grp .. for 64) of entries 2 tig, 2 tig + 1, 2 tig + 8, 2 tig + 9
#pragma unroll
            for (int xt = 0; xt < ET; ++xt) {
                uint32_t v[4][DH / 32];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 16 * xt + 2 * tig + (e & 1) + (e >> 1) * 8;
                    if (DH == 128) {
                        const uint4 x = *reinterpret_cast<const uint4*>(vs_s + few_v_off<DH>(r, grp));
                        v[e][0] = x.x;
                        v[e][1] = x.y;
                        v[e][DH / 32 - 2] = x.z;
                        v[e][DH / 32 - 1] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2*>(vs_s + few_v_off<DH>(r, grp >> 1) + (grp & 1) * 8);
                        v[e][0] = x.x;
                        v[e][1] = x.y;
                    }
                }
#pragma unroll
                for (int i = 0; i < DH / 32; ++i) {
                    // bytes of two entries side by side: (dim 0, dim 1), (dim 2, dim 3)
                    const uint32_t x0 = __byte_perm(v[0][i], v[1][i], 0x5140), x1 = __byte_perm(v[0][i], v[1][i], 0x7362);
                    const uint32_t y0 = __byte_perm(v[2][i], v[3][i], 0x5140), y1 = __byte_perm(v[2][i], v[3][i], 0x7362);
                    const uint32_t a0 = decode_lo(x0), a1 = decode_hi(x0), a2 = decode_lo(y0), a3 = decode_hi(y0);
                    const uint32_t b0 = decode_lo(x1), b1 = decode_hi(x1), b2 = decode_lo(y1), b3 = decode_hi(y1);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        mma_f16(o[t][2 * i], a0, a1, a2, a3, pb[xt][t][0], pb[xt][t][1]);
                        mma_f16(o[t][2 * i + 1], b0, b1, b2, b3, pb[xt][t][0], pb[xt][t][1]);
                    }
                }
            }
        }
        // ---- the warps' outputs, joined: of eight warps 4 .. 7 hand theirs to 0 .. 3, and four are added up in order
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) l[t][h] += __shfl_xor_sync(0xffffffffu, l[t][h], w);
                const PartRef ref = part_ref(m[t][h], v_ref[t][h], l[t][h]);
                m[t][h] = ref.m;
                l[t][h] = ref.l;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    o[t][i][h] *= ref.by;
                    o[t][i][2 + h] *= ref.by;
                }
            }
        const bool whole = it.whole();
        float* part = reinterpret_cast<float*>(p.scratch + part_off) + ((size_t)me * 2 + (it.kv0 == 0 ? 1 : 0)) * part_floats(part_rows, DH);
        const int first_row = it.q0 + i0, g = it.g;
        if (it.begun() && threadIdx.x == 0)
            reinterpret_cast<SharedItem*>(p.scratch)[me] = {first_row, rows, g, it.last_worker(piece[0])};
        it.next(c, shape);
        load_queries();
        float* my_o = join_s + (size_t)(warp & 3) * ROWS * DH;
        float* my_ml = join_s + (size_t)4 * ROWS * DH + (warp & 3) * ROWS * 2;
        auto leave = [&]() {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = t * 8 + 2 * tig + h;
#pragma unroll
                    for (int i = 0; i < MT; i += 2)  // four dims: (i, 0), (i, 2), (i + 1, 0), (i + 1, 2)
                        *reinterpret_cast<float4*>(my_o + few_join_at<DH>(r, grp * (MT / 2) + i / 2)) =
                            make_float4(o[t][i][h], o[t][i][2 + h], o[t][i + 1][h], o[t][i + 1][2 + h]);
                    if (grp == 0) *reinterpret_cast<float2*>(my_ml + 2 * r) = make_float2(m[t][h], l[t][h]);
                }
        };
        if (WARPS > 4) {
            if (warp >= 4) leave();
            __syncthreads();
        }
        if (WARPS == 4) {
            leave();
        } else if (warp < 4) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = t * 8 + 2 * tig + h;
                    const float2 e = *reinterpret_cast<const float2*>(my_ml + 2 * r);
                    const float now = fmaxf(m[t][h], e.x), ref = now == -INFINITY ? 0.f : now;
                    const float f = exp2f(m[t][h] - ref), w = exp2f(e.x - ref);
                    m[t][h] = now;
                    l[t][h] = l[t][h] * f + e.y * w;
#pragma unroll
                    for (int i = 0; i < MT; i += 2) {
                        const float4 x = *reinterpret_cast<const float4*>(my_o + few_join_at<DH>(r, grp * (MT / 2) + i / 2));
                        o[t][i][h] = o[t][i][h] * f + x.x * w;
                        o[t][i][2 + h] = o[t][i][2 + h] * f + x.y * w;
                        o[t][i + 1][h] = o[t][i + 1][h] * f + x.z * w;
                        o[t][i + 1][2 + h] = o[t][i + 1][2 + h] * f + x.w * w;
                    }
                }
            __syncwarp();
            leave();
        }
        __syncthreads();
        const float* ml = join_s + (size_t)4 * ROWS * DH;
        for (int i = threadIdx.x; i < rows * (DH / 4); i += THREADS) {
            const int r = i / (DH / 4), d = i % (DH / 4) * 4;
            float2 e[4];
            float M = -INFINITY, L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                e[w] = *reinterpret_cast<const float2*>(ml + (w * ROWS + r) * 2);
                M = fmaxf(M, e[w].x);
            }
            const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = exp2f(e[w].x - ref);
                const float4 y = *reinterpret_cast<const float4*>(join_s + (size_t)w * ROWS * DH + few_join_at<DH>(r, d / 4));
                L += e[w].y * f;
                x[0] += y.x * f;
                x[1] += y.y * f;
                x[2] += y.z * f;
                x[3] += y.w * f;
            }
            if (whole) {
                const float inv = L > 0.f ? 1.f / L : 0.f;
                const int t = r / c.G;
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] *= inv;
                store_f<bf16_t, 4>(static_cast<bf16_t*>(p.out) + (size_t)(first_row + t) * p.ld_out +
                                       (size_t)(g * c.G + r - t * c.G) * DH + d,
                                   x);
            } else {
                *reinterpret_cast<float4*>(part + ((size_t)(d / 4) * part_rows + r) * 4) = make_float4(x[0], x[1], x[2], x[3]);
                if (d == 0) *reinterpret_cast<float2*>(part + (size_t)part_rows * DH + 2 * r) = make_float2(M, L);
            }
        }
        __syncthreads();  // the joining memory is read
    }
    cp_async_wait<0>();
}

}  // namespace pipo
