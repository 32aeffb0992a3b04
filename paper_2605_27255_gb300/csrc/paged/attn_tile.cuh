// Attention of ragged chunks over a paged bf16 cache on the tensor cores
// (tcgen05, sm_103a).
//
// out = softmax(scale Q K^T) V for row tiles of 128 rows (tokens times the query
// heads of one kv head), the rows of the MMAs, over 64 cache entries at a time:
//   S = Q K^T   fp32 in TMEM, Q and K from shared memory (K-major);
//   softmax     one thread per row: it reads the row's 64 scores, keeps the
//               running maximum and sum in fp32, and writes exp2 of the scores back over
//               them as bf16 (the A operand of the next MMAs, from TMEM); their sum
//               is taken before the rounding.  PAIR (below): one part, whose 2^-9 of a
//               weight is about the output's own rounding (together 1.4 times
//               its error).  Single: bf16 part and bf16 remainder, since the MMAs have time
//               under the pages' copies; the output's rounding is then all there is;
//   O += P V    fp32 in TMEM over the whole item; V is the [entry][dim] tile as it
//               lies in the cache (MN-major).  The reference that the
//               exponents are taken against moves only when the running maximum
//               has passed it by 2^8: until then the weights are at most 256 and
//               neither O nor the sum is touched; when it moves the row's
//               thread rescales its row of O in TMEM.
// (Such a reference, and warps of their own for issuing, softmax and copies, are published
// methods for attention on this architecture.)
//
// The scores of 64 entries (a page) have a buffer each, two per pipeline, so that
// the softmax of one page runs under the MMAs of the next: with one buffer of 128
// entries every unit waits for its own chain of scores, softmax and values (429 us for a
// 2048-token chunk over 16 K entries).  The price is that an MMA of 64 columns is bound by
// shared memory (A and B rows: 48 cycles against 32).
//
// A CTA runs two such pipelines side by side:
//   PAIR    the two halves of a 256-row tile: both read each K and V tile
//           (one copy, two uses).  Chunks of many rows.
//   single  two workers with items of their own (work.cuh), 128 rows each, and a
//           ring of copies each.  Few rows per sequence, listed pages.
//
// Roles (512 threads): warps 0 and 2 copy K and V tiles (TMA boxes of one page x
// 64 dims, 128-byte swizzle; PAIR: warp 0 alone), warps 1 and 3 issue the score
// MMAs of the two pipelines, warps 13 and 15 their value MMAs, and warps 4-7 and 8-11 are
// the two softmax warpgroups, which also load the queries and write the
// outputs.  Scores and values have issuing warps of their own because a warp's next
// wait is held until its MMAs have left the queue (about 250 cycles each: 440 us
// for the 2048-token chunk with one warp for both).  Cache slots past a
// sequence's end or before its window may hold anything: their scores are masked, and the value warp
// clears their values in shared memory (0 times NaN would be NaN).
//
// Bound and measured (32 query and 8 kv heads of 128): 2048 tokens behind 14336 entries, 388 us,
// 1.33 PFLOP/s, by the score MMAs' shared-memory reads and the softmax's latency; four
// sequences of 15.5 K entries with one token each, 53.9 us with the joining, 4.7 TB/s (35 us of
// them the pages' stream at HBM rate).
//
// Every wait is bounded; when one gives up the error word is set, every role
// stops, and the copies and commits in flight are waited for before the CTA ends.
#pragma once

#include <cuda_fp16.h>

#include "../attn_prefill.cuh"
#include "codes.cuh"
#include "work.cuh"

namespace pipo {

constexpr int kAtThreads = 512;
constexpr int kAtRegsIo = 72, kAtRegsSoft = 184;  // (56 and 200: 396 us for the 2048-token chunk, these 389)
static_assert(2 * kAtRegsIo + 2 * kAtRegsSoft <= 4 * 128, "register shares must fit the launch's registers");
constexpr int kAtHalf = 128 * 128;      // 64 dims of a query tile: 128 rows of 128 bytes
constexpr int kPageHalf = kPage * 128;  // 64 dims of a page
constexpr float kAtSlack = 8.f;         // exponents above the reference before it moves

__host__ __device__ constexpr int at_q_bytes(int dh) { return dh / 64 * kAtHalf; }
__host__ __device__ constexpr int at_page_bytes(int dh) { return dh / 64 * kPageHalf; }
// Pages in a ring of K and in one of V (single: each pipeline has its own two).  Separate
// rings: the score warps wait for every K page in turn and the value warps for every V
// page, so that a parity always tells a fill from the one before it.
__host__ __device__ constexpr int at_k_pages(int dh, bool pair) { return pair ? (dh == 128 ? 5 : 8) : (dh == 128 ? 3 : 6); }
__host__ __device__ constexpr int at_v_pages(int dh, bool pair) { return pair ? (dh == 128 ? 5 : 8) : (dh == 128 ? 2 : 6); }
__host__ __device__ constexpr size_t at_smem(int dh, bool pair) {
    return 1024 + 2 * (size_t)at_q_bytes(dh) +
           (size_t)at_page_bytes(dh) * (at_k_pages(dh, pair) + at_v_pages(dh, pair)) * (pair ? 1 : 2);
}

// 8-bit pools: pages of key codes, of value operands and of value codes on their way to those, in a ring each
// (single: per pipeline)
__host__ __device__ constexpr int at8_k_pages(int dh, bool pair) { return pair ? (dh == 128 ? 7 : 8) : (dh == 128 ? 2 : 6); }
__host__ __device__ constexpr int at8_v_pages(int dh, bool pair) { return pair ? (dh == 128 ? 3 : 6) : (dh == 128 ? 2 : 4); }
__host__ __device__ constexpr int at8_raw_pages(int dh, bool pair) { return pair ? (dh == 128 ? 3 : 9) : (dh == 128 ? 2 : 4); }
__host__ __device__ constexpr int at8_q_bytes(int dh) { return 3 * 128 * dh; }  // three parts of a query tile
__host__ __device__ constexpr int at8_convert(bool pair) { return pair ? 3 : 1; }  // converting warps of a ring
__host__ __device__ constexpr int at8_codes(int dh) { return kPage * dh; }
__host__ __device__ constexpr int at8_ring_bytes(int dh, bool pair) {
    return at_page_bytes(dh) * at8_v_pages(dh, pair) + at8_codes(dh) * (at8_k_pages(dh, pair) + at8_raw_pages(dh, pair));
}
__host__ __device__ constexpr size_t at8_smem(int dh, bool pair) {
    return 1024 + 2 * (size_t)at8_q_bytes(dh) + (size_t)at8_ring_bytes(dh, pair) * (pair ? 1 : 2);
}

// B operand [entries][dims] of a page (MN-major, 128-byte swizzle): 64-dim blocks kPageHalf apart,
// groups of 8 entries 1024 bytes apart
__device__ __forceinline__ uint64_t umma_desc_mn_page(uint32_t saddr) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
    d |= (uint64_t)(kPageHalf >> 4) << 16;  // leading byte offset: next 64 dims
    d |= (uint64_t)(1024 >> 4) << 32;       // stride byte offset: next 8 entries
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// K-major with 64-byte rows: 64-byte swizzle, 8-row groups 512 bytes apart
__device__ __forceinline__ uint64_t umma_desc_sw64(uint32_t saddr) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
    d |= (uint64_t)1 << 16;
    d |= (uint64_t)(512 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)4 << 61;  // 64-byte swizzle
    return d;
}

// D += A B of e4m3 numbers from shared memory, 32 bytes of a row at a time
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}" ::"r"(
            d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}

// x / G for x < 256 and G <= 16, magic = ceil(2^16 / G): off by less than 256 / 2^16 < 1 / G
__device__ __forceinline__ int div_g(int x, uint32_t magic) { return (int)(((uint32_t)x * magic) >> 16); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// one thread of the converged warp, always the same one (the compiler knows that it is alone, which a
// test of the lane does not tell it: 75 cycles less for every eight MMAs)
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
    return e != 0;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ float max32(const uint32_t (&s)[32]) {
    float a = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])), b = fmaxf(__uint_as_float(s[2]), __uint_as_float(s[3]));
#pragma unroll
    for (int j = 4; j < 32; j += 4) {
        a = max3(a, __uint_as_float(s[j]), __uint_as_float(s[j + 1]));
        b = max3(b, __uint_as_float(s[j + 2]), __uint_as_float(s[j + 3]));
    }
    return fmaxf(a, b);
}

// pairs of fp32 values, the first one in the low word
__device__ __forceinline__ uint64_t u32x2(uint32_t a, uint32_t b) { return (uint64_t)b << 32 | a; }
__device__ __forceinline__ uint64_t f32x2(float a, float b) { return u32x2(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// 32 consecutive fp32 columns of this thread's TMEM lane, without the wait
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,"
        "%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// the loaded values exist from here on: nothing may use them before the wait
__device__ __forceinline__ void pin32(uint32_t (&r)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(r[i]));
}

// The codes of a page as an fp16 operand tile: rows of 64 entries, dims in blocks of 64, 128-byte
// swizzle.  A quarter of the warp takes half of two neighbouring rows (128-dim rows: opposite halves), so that
// neither its loads nor its stores meet in a bank.  How much is unrolled decides over the whole kernel's time,
// whose warps wait for instructions (1.6 of the 9 cycles between two of them, against 0.7 in the bf16 kernel): the
// 2048-token chunk takes 488 us with one group of rows in flight, 472 with two, 449 with four, 517 with eight.
template <int DH>
__device__ __forceinline__ void page_from_codes(unsigned char* dst, const unsigned char* src) {
    constexpr int U = 4, H = DH / 64;  // groups of eight rows in flight, halves of a row
    const int lane = threadIdx.x & 31, sub = lane >> 2 & 1, quad = lane & 3, r = (lane >> 3) * 2 + sub;  // row of a group
    uint32_t from[H], to[H][2];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int half = DH == 128 ? sub ^ h : 0;
        from[h] = smem_u32(src) + r * DH + half * 64 + quad * 16;
#pragma unroll
        for (int k = 0; k < 2; ++k) to[h][k] = smem_u32(dst) + half * kPageHalf + r * 128 + (((2 * quad + k) ^ r) << 4);
    }
#pragma unroll 1
    for (int g = 0; g < kPage / 8; g += U) {
        uint4 x[U][H];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < H; ++h)
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(x[u][h].x), "=r"(x[u][h].y), "=r"(x[u][h].z), "=r"(x[u][h].w)
                             : "r"(from[h] + u * 8 * DH));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const uint4 y = x[u][h];
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to[h][0] + u * 1024), "r"(decode_lo(y.x)),
                             "r"(decode_hi(y.x)), "r"(decode_lo(y.y)), "r"(decode_hi(y.y))
                             : "memory");
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to[h][1] + u * 1024), "r"(decode_lo(y.z)),
                             "r"(decode_hi(y.z)), "r"(decode_lo(y.w)), "r"(decode_hi(y.w))
                             : "memory");
            }
#pragma unroll
        for (int h = 0; h < H; ++h) {
            from[h] += U * 8 * DH;
            to[h][0] += U * 1024;
            to[h][1] += U * 1024;
        }
    }
}

// SEL: whole tiles over selected pages (AttnPagedArgs::bits), PAIR only.
// E8: pools of e4m3 codes.  Key codes are operands as they are (kind::f8f6f4): queries are scaled
// by a power of two per row to below 2^15 and meet them as three e5m2 parts of three digits each (the
// rest of the one before, so that its sign is a digit too): all digits of a bf16 number down to 2^-24 of the row's
// largest, and what is below 2^-31 of that is lost.  (Two e4m3 parts cost a third less and hold 2^-10 and 2^-18: a row
// whose other dims lie 2^10 below one that the keys do not have is then off by more than the output's
// rounding.)  The row's and the block's scale meet the
// scores in fp32.  Value codes become fp16 tiles (a code is an fp16 number) by warps 2, 12 and 14 (single: 12 and
// 14, one per pipeline); their scales go into the weights (codes.cuh), which keep fp16's 11 digits.
// (Weights as e4m3 parts, so that values need no conversion either, would lose the small ones: a
// long tail of 2^-17 each next to one large weight.)  Measured for 2048 tokens behind 14336 entries, 32
// query and 8 kv heads of 128: 2559 us with row tiles of 32 on mma.sync, 692 with keys converted too (by two
// warps; 592 by three), 541 with key codes as operands, 465 with the scales by shuffles in place of a
// barrier, 445 with fixed addresses in the conversion, 475 with the queries' third part (492 with rings of 5, 4 and 3
// pages of keys, values and value codes in the shared memory it leaves, 484 with 4, 3 and 6; 7, 3 and 3 are taken); the
// bf16 pools take 375.  What is left: instruction fetch, the scales' part of every page (20 us), the key products (three
// parts take half as long again as the bf16 kernel's).
template <int DH, bool PAIR, bool SEL, bool E8 = false>
__global__ void __launch_bounds__(kAtThreads, 1) attn_tile_kernel(AttnPagedArgs p, ItemShape shape, int S,
                                                                  int part_rows, size_t part_off,
                                                                  const __grid_constant__ CUtensorMap tmK,
                                                                  const __grid_constant__ CUtensorMap tmV) {
    constexpr int kTile = E8 ? at8_q_bytes(DH) : at_q_bytes(DH), kPg = at_page_bytes(DH), NR = PAIR ? 1 : 2;  // NR: pairs of rings
    constexpr int PARTS = PAIR || E8 ? 1 : 2;  // parts of the weights
    constexpr int SK = E8 ? at8_k_pages(DH, PAIR) : at_k_pages(DH, PAIR), SV = E8 ? at8_v_pages(DH, PAIR) : at_v_pages(DH, PAIR);
    constexpr int SR = at8_raw_pages(DH, PAIR), kCodes = at8_codes(DH);
    static_assert(!E8 || !SEL, "selected pages: bf16 pools");
    extern __shared__ __align__(1024) unsigned char at_smem_raw[];
    __shared__ uint32_t tmem_base;
    __shared__ __align__(8) uint64_t k_full[NR][SK], k_empty[NR][SK], v_full[NR][SV], v_empty[NR][SV];
    __shared__ __align__(8) uint64_t q_full[2], s_full[2][2], p_full[2][2], o_full[2][2], drained[4];
    __shared__ Piece pieces[NR];
    __shared__ int give_up;
    // 8-bit pools: ring of value codes, the queries' row scales
    __shared__ __align__(8) uint64_t raw_full[E8 ? NR : 1][E8 ? SR : 1], raw_empty[E8 ? NR : 1][E8 ? SR : 1];
    __shared__ bool raw_live[E8 ? NR : 1][E8 ? SR : 1];
    __shared__ int8_t row_scale[E8 ? 2 : 1][E8 ? 2 : 1][E8 ? 128 : 1];  // [item's parity][pipeline][row], exponents of two

    unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(at_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* q_s = sm;              // two query tiles
    unsigned char* ring_s = sm + 2 * kTile;  // NR times SK pages of K, SV pages of V

    const PagedArgs& c = p.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 0) tmem_alloc(&tmem_base, 512);
    if (threadIdx.x == 32) {
        prefetch_tmap(&tmK);
        prefetch_tmap(&tmV);
        for (int r = 0; r < NR; ++r) {  // (an empty barrier counts the pipelines that read a page)
            for (int i = 0; i < SK; ++i) {
                mbar_init(&k_full[r][i], 1);
                mbar_init(&k_empty[r][i], PAIR ? 2 : 1);
            }
            for (int i = 0; i < SV; ++i) {
                mbar_init(&v_full[r][i], 1);
                mbar_init(&v_empty[r][i], PAIR ? 2 : 1);
            }
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(q_full + w, 4);  // softmax warps
            for (int i = 0; i < 2; ++i) {
                mbar_init(&s_full[w][i], 1);
                mbar_init(&p_full[w][i], 4);
                mbar_init(&o_full[w][i], 1);  // by the page's buffer too: with one barrier a late waiter could miss a phase
            }
            mbar_init(drained + 2 * w, 1);
            mbar_init(drained + 2 * w + 1, 1);
        }
        if (E8) {
            for (int r = 0; r < NR; ++r)
                for (int i = 0; i < SR; ++i) {
                    mbar_init(&raw_full[r][i], 1);
                    mbar_init(&raw_empty[r][i], 1);
                }
        }
        give_up = 0;
        mbar_init_fence();
    }
    pdl_wait();  // lengths, queries, entries and the scratch come from the kernels before
    // (the sequences' tile counts use the ring's memory before any copy)
    find_pieces<kAtThreads, NR>(c, shape, (int)blockIdx.x * NR, S, reinterpret_cast<int*>(ring_s), pieces);
    fence_proxy_async();  // those generic accesses, before the copies into the ring
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch();  // after the allocation: a dependent CTA must not take this SM's TMEM first
    const uint32_t tmem = tmem_base;

    // bounded wait of a whole warp that stops every role of the CTA once it gives up
    auto wait = [&](uint64_t* bar, uint32_t parity, unsigned site, int it) -> bool {
        bool got = mbar_try_wait(bar, parity);
        if (!got && !*(volatile int*)&give_up) got = mbar_wait(bar, parity, site, (unsigned)it);
        got = __all_sync(0xffffffffu, got);
        if (!got) *(volatile int*)&give_up = 1;
        return got;
    };

    if (warp < 4 || warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kAtRegsIo));
        const int chain = (warp >> 1) & 1, ring = PAIR ? 0 : chain;  // PAIR: one ring for both pipelines, filled by warp 0
        if ((warp & 1) ? true : warp < 4 && !(PAIR && warp == 2)) {
            ItemWalk it;
            it.start(c, shape, pieces[ring]);
            // (8-bit pools: value operands, key codes, value codes)
            unsigned char* k_s = E8 ? ring_s + ring * at8_ring_bytes(DH, PAIR) + SV * kPg : ring_s + (size_t)ring * (SK + SV) * kPg;
            unsigned char* v_s = E8 ? k_s - SV * kPg : k_s + SK * kPg;
            if (E8 && (warp & 1) == 0) {
                // ---- copies of codes: the keys one page ahead of the values
                unsigned char* raw_s = k_s + SK * kCodes;
                int kn = 0, vn = 0;  // pages issued
                bool ok = true;
                for (; it.more() && ok; it.next(c, shape)) {
                    const int np = it.pages(), pg0 = (it.t0 + it.kv0) * 2;
                    const int gone = first_seen(shape, it.n, it.len, it.tile) / kPage;  // pages that no row sees
                    int held = -32, mine = -1, prev = -1;  // lane l holds the block of page held + l
                    for (int j = 0; j <= np; ++j) {
                        int blk = -1;
                        if (j < np) {
                            if (j >= held + 32) {
                                held = j;
                                const int i = pg0 + j + lane;
                                mine = j + lane < np && i * kPage < it.len && i >= gone ? page_block(c, it.b, i) : -1;
                            }
                            blk = __shfl_sync(0xffffffffu, mine, j - held);
                            const int st = kn % SK;
                            ok = kn < SK || wait(&k_empty[ring][st], (uint32_t)(((kn / SK) & 1) ^ 1), 51, kn);
                            if (!ok) break;
                            if (lane == 0) {
                                if (blk < 0) {
                                    mbar_arrive(&k_full[ring][st]);
                                } else {
                                    mbar_arrive_expect_tx(&k_full[ring][st], (uint32_t)kCodes);
                                    tma_load_2d(k_s + st * kCodes, &tmK, 0, (blk * c.n_kv + it.g) * kPage, &k_full[ring][st]);
                                }
                            }
                            ++kn;
                            __syncwarp();
                        }
                        if (j > 0) {
                            const int st = vn % SR;
                            ok = vn < SR || wait(&raw_empty[ring][st], (uint32_t)(((vn / SR) & 1) ^ 1), 51, vn);
                            if (!ok) break;
                            if (lane == 0) {
                                raw_live[ring][st] = prev >= 0;
                                if (prev < 0) {
                                    mbar_arrive(&raw_full[ring][st]);
                                } else {
                                    mbar_arrive_expect_tx(&raw_full[ring][st], (uint32_t)kCodes);
                                    tma_load_2d(raw_s + st * kCodes, &tmV, 0, (prev * c.n_kv + it.g) * kPage, &raw_full[ring][st]);
                                }
                            }
                            ++vn;
                            __syncwarp();
                        }
                        prev = blk;
                    }
                }
                if (lane == 0) {
                    ring_drain<SK>(kn, [&](int st, uint32_t ph, int i) { mbar_wait(&k_full[ring][st], ph, 52, (unsigned)i); });
                    ring_drain<SR>(vn, [&](int st, uint32_t ph, int i) { mbar_wait(&raw_full[ring][st], ph, 52, (unsigned)i); });
                }
            } else if ((warp & 1) == 0) {
                // ---- copies: the keys one page ahead of the values
                int kn = 0, vn = 0;  // pages issued
                bool ok = true;
                for (; it.more() && ok; it.next(c, shape)) {
                    const int32_t* list =
                        shape.n_top > 0 ? p.pages + ((size_t)(it.q0 + it.tile) * c.n_kv + it.g) * shape.n_top : nullptr;
                    const int np = it.pages(), pg0 = (it.t0 + it.kv0) * 2;  // first page in the cache or the list
                    const int gone = first_seen(shape, it.n, it.len, it.tile) / kPage;  // pages that no row sees
                    int held = -32, mine = -1;  // lane l holds the block of page held + l
                    int prev = -1;              // block of the page whose values come next
                    for (int j = 0; j <= np; ++j) {
                        int blk = -1;
                        if (j < np) {
                            if (j >= held + 32) {
                                held = j;
                                const int i = pg0 + j + lane;
                                if (list) {
                                    const int q = i < shape.n_top ? list[i] : -1;
                                    mine = q >= 0 ? page_block(c, it.b, q) : -1;
                                } else {
                                    mine = j + lane < np && i * kPage < it.len && i >= gone ? page_block(c, it.b, i) : -1;
                                }
                            }
                            blk = __shfl_sync(0xffffffffu, mine, j - held);
                        }
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            if (v ? j == 0 : j == np) continue;
                            const int n = v ? vn : kn, S_ = v ? SV : SK, st = n % S_, from = v ? prev : blk;
                            uint64_t* fu = v ? &v_full[ring][st] : &k_full[ring][st];
                            ok = n < S_ || wait(v ? &v_empty[ring][st] : &k_empty[ring][st], (uint32_t)(((n / S_) & 1) ^ 1), 51, n);
                            if (!ok) break;
                            if (lane == 0) {
                                if (from < 0) {
                                    mbar_arrive(fu);
                                } else {
                                    mbar_arrive_expect_tx(fu, (uint32_t)kPg);
#pragma unroll
                                    for (int d = 0; d < DH / 64; ++d)
                                        tma_load_2d((v ? v_s : k_s) + st * kPg + d * kPageHalf, v ? &tmV : &tmK, d * 64,
                                                    (from * c.n_kv + it.g) * kPage, fu);
                                }
                            }
                            if (v) ++vn; else ++kn;
                        }
                        __syncwarp();
                        if (!ok) break;
                        prev = blk;
                    }
                }
                // no copy into this CTA's shared memory is in flight at its end
                if (lane == 0) {
                    ring_drain<SK>(kn, [&](int st, uint32_t ph, int i) { mbar_wait(&k_full[ring][st], ph, 52, (unsigned)i); });
                    ring_drain<SV>(vn, [&](int st, uint32_t ph, int i) { mbar_wait(&v_full[ring][st], ph, 52, (unsigned)i); });
                }
            } else {
                // ---- MMAs.  TMEM: scores / weights of pipeline w at w * 128 (two buffers of 64 columns),
                // its output at 256 + w * 128
                const bool values = warp >= 12;  // this warp's half of them
                int items = 0;    // items begun
                int n = 0;        // pages of K or V taken from the ring
                int pv = 0;       // pages of this pipeline
                bool ok = true;
                const uint32_t s_at = tmem + (uint32_t)(chain * 128), o_at = s_at + 256u;
                auto filled = [&](int i) {
                    return values ? wait(&v_full[ring][i % SV], (uint32_t)((i / SV) & 1), 54, i)
                                  : wait(&k_full[ring][i % SK], (uint32_t)((i / SK) & 1), 54, i);
                };
                for (; it.more() && ok; it.next(c, shape)) {
                    const int np = it.pages();
                    if (PAIR && chain * 128 >= it.tokens(shape) * c.G) {  // no rows here: hand the pages on
                        for (int j = 0; j < np && ok; ++j, ++n) {
                            ok = filled(n);
                            if (ok && lane == 0) mbar_arrive(values ? &v_empty[ring][n % SV] : &k_empty[ring][n % SK]);
                        }
                        continue;
                    }
                    if (!values) {
                        constexpr uint32_t id_s = E8 ? umma_idesc_e5m2_e4m3(128, kPage) : umma_idesc_bf16(128, kPage);
                        // descriptors count in 16 bytes: a step along a tile is an addition
                        constexpr int kPgK = E8 ? kCodes : kPg;
                        const uint32_t q_at = smem_u32(q_s) + chain * kTile, k_at = smem_u32(k_s);
                        const uint64_t dq = E8 && DH == 64 ? umma_desc_sw64(q_at) : umma_desc_sw128(q_at);
                        const uint64_t dk = E8 && DH == 64 ? umma_desc_sw64(k_at) : umma_desc_sw128(k_at);
                        ok = wait(q_full + chain, (uint32_t)(items & 1), 53, items);
                        for (int j = 0; j < np && ok; ++j, ++pv, ++n) {
                            const int st = n % SK, buf = pv & 1;
                            // the weights of the page before last lie in the buffer until their values are done
                            ok = filled(n) && (pv < 2 || wait(&o_full[chain][buf], (uint32_t)(((pv - 2) >> 1) & 1), 56, pv));
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                uint32_t qb = (uint32_t)dq, kb = (uint32_t)dk + (uint32_t)((st * kPgK) >> 4);
                                asm volatile("" : "+r"(qb), "+r"(kb));  // eight sums now, not sixteen kept over the loop
                                if constexpr (E8) {  // 32 dims a step; the queries' parts lie one behind the other
#pragma unroll
                                    for (int i = 0; i < 3 * DH / 32; ++i)
                                        umma_f8(s_at + buf * 64,
                                                u32x2(qb + ((i / (DH / 32) * 128 * DH + i % (DH / 32) * 32) >> 4), (uint32_t)(dq >> 32)),
                                                u32x2(kb + ((i % (DH / 32) * 32) >> 4), (uint32_t)(dk >> 32)), id_s, i > 0 ? 1u : 0u);
                                } else
#pragma unroll
                                for (int i = 0; i < DH / 16; ++i)
                                    umma_bf16(s_at + buf * 64,
                                              u32x2(qb + (((i >> 2) * kAtHalf + (i & 3) * 32) >> 4), (uint32_t)(dq >> 32)),
                                              u32x2(kb + (((i >> 2) * kPageHalf + (i & 3) * 32) >> 4), (uint32_t)(dk >> 32)), id_s,
                                              i > 0 ? 1u : 0u);
                                umma_commit(&s_full[chain][buf]);
                                umma_commit(&k_empty[ring][st]);
                            }
                            __syncwarp();
                        }
                    } else {
                        constexpr uint32_t id_o = (E8 ? umma_idesc_f16(128, DH) : umma_idesc_bf16(128, DH)) | (1u << 16);  // B MN-major
                        const uint64_t dv = umma_desc_mn_page(smem_u32(v_s));
                        // entries whose values may be anything: those before the window and past the
                        // sequence's (or the list's) end
                        const int first = first_seen(shape, it.n, it.len, it.tile);
                        int end = it.len;
                        if (shape.n_top > 0) {
                            const int pos = it.len - it.n + it.tile;
                            const int kept = pos < 0 ? 0 : min(shape.n_top, pos / kPage + 1);
                            const int32_t* list = p.pages + ((size_t)(it.q0 + it.tile) * c.n_kv + it.g) * shape.n_top;
                            end = kept == 0 ? 0 : (kept - 1) * kPage + (list[kept - 1] == pos / kPage ? pos % kPage + 1 : kPage);
                        }
                        for (int j = 0; j < np; ++j, ++pv, ++n) {
                            const int st = n % SV, buf = pv & 1;
                            ok = filled(n);
                            if (!ok) break;
                            const int at = (it.t0 + it.kv0) * kTileEnt + j * kPage, head = min(kPage, first - at), tail = end - at;
                            if (head > 0 || tail < kPage) {  // (PAIR: both pipelines clear the same rows before their own MMAs)
                                const int a = max(0, head), z = min(kPage - a, kPage - max(0, tail));  // rows before, rows past
                                for (int i = lane; i < (a + max(0, z)) * (DH / 8); i += 32) {
                                    int r = i / (DH / 8);
                                    const int ch = i % (DH / 8);
                                    r = r < a ? r : kPage - 1 - (r - a);
                                    *reinterpret_cast<uint4*>(v_s + st * kPg + (ch >> 3) * kPageHalf + r * 128 + (ch & 7) * 16) =
                                        make_uint4(0u, 0u, 0u, 0u);
                                }
                                fence_proxy_async();
                                __syncwarp();
                            }
                            ok = wait(&p_full[chain][buf], (uint32_t)((pv >> 1) & 1), 55, pv);
                            if (!ok) break;
                            tc_fence_after();
                            if (elect_one()) {
                                uint32_t vb = (uint32_t)dv + (uint32_t)((st * kPg) >> 4);
                                asm volatile("" : "+r"(vb));
#pragma unroll
                                for (int i = 0; i < PARTS * kPage / 16; ++i)  // (the second part lies behind the first)
                                    umma_bf16_ta(o_at, s_at + buf * 64 + i * 8,
                                                 u32x2(vb + i % (kPage / 16) * (2048 >> 4), (uint32_t)(dv >> 32)), id_o,
                                                 i > 0 || j > 0 ? 1u : 0u);
                                umma_commit(&o_full[chain][buf]);
                                umma_commit(&v_empty[ring][st]);
                            }
                            __syncwarp();
                        }
                    }
                    ++items;
                }
                // commits arrive in order: after one more, none is in flight at the CTA's end
                if (elect_one()) {
                    umma_commit(drained + 2 * chain + values);
                    mbar_wait(drained + 2 * chain + values, 0, 57);
                }
            }
        } else if (E8) {
            // ---- value codes to operands: the converting warps take the pages in turn, each from stages of its own
            ItemWalk it;
            const int rg = PAIR ? 0 : (warp - 12) >> 1, me = PAIR ? (warp == 2 ? 2 : (warp - 12) >> 1) : 0;
            constexpr int W = at8_convert(PAIR);
            static_assert(ring_turns_ok(SR, W) && ring_fillers_ok(SV, W), "parities of the rings that the converting warps share");
            it.start(c, shape, pieces[rg]);
            unsigned char *v_s = ring_s + rg * at8_ring_bytes(DH, PAIR), *raw_s = v_s + SV * kPg + SK * kCodes;
            int n = 0;  // pages before the present item
            bool ok = true;
            for (; it.more() && ok; it.next(c, shape)) {
                const int end = n + it.pages();
                for (int i = n + (me + W - n % W) % W; i < end; i += W) {
                    const int st = i % SR, to = i % SV;
                    ok = wait(&raw_full[rg][st], (uint32_t)((i / SR) & 1), 61, i) &&
                         (i < SV || wait(&v_empty[rg][to], (uint32_t)(((i / SV) & 1) ^ 1), 62, i));
                    if (!ok) break;
                    if (raw_live[rg][st]) page_from_codes<DH>(v_s + to * kPg, raw_s + st * kCodes);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&v_full[rg][to]);
                        mbar_arrive(&raw_empty[rg][st]);
                    }
                    __syncwarp();
                }
                n = end;
            }
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kAtRegsSoft));
        // ---- softmax warpgroup w: thread = row r of its tile
        const int w = (warp - 4) >> 2, quad = warp & 3, r = quad * 32 + lane, wt = threadIdx.x - 128 - w * 128;
        const uint32_t lane_addr = tmem + ((uint32_t)(quad * 32) << 16);
        const uint32_t s_col = lane_addr + (uint32_t)(w * 128), o_col = lane_addr + 256u + (uint32_t)(w * 128);
        const int me = (int)blockIdx.x * NR + (PAIR ? 0 : w);
        const float c2 = p.scale * 1.4426950408889634f;  // exponents of two
        ItemWalk it;
        it.start(c, shape, pieces[PAIR ? 0 : w]);
        const uint32_t g_magic = (65536u + (uint32_t)c.G - 1) / (uint32_t)c.G;
        const int row0 = PAIR ? w * 128 : 0;
        int begun = 0;  // 8-bit pools: items with queries loaded
        // the next item with rows for this warpgroup, its queries in shared memory (rows past the last one
        // are zero).  Every load is in flight before the first is stored (one after the other they
        // took 19000 cycles).
        auto queries = [&]() {
            if (PAIR)
                while (it.more() && it.tokens(shape) * c.G <= row0) it.next(c, shape);
            if (!it.more()) return;
            constexpr int C = DH / 8, RS = 128 / C, NI = 128 / RS;  // 16-byte chunks a row, rows per round, rounds
            const int ch = wt % C, v0 = wt / C, rows = it.tokens(shape) * c.G - row0;
            const bf16_t* q = static_cast<const bf16_t*>(p.q) + (size_t)(it.q0 + it.tile * shape.TP) * p.ld_q +
                              (size_t)it.g * c.G * DH + ch * 8;
            auto load = [&](int v) {
                const int t = div_g(row0 + v, g_magic);
                return v < rows ? *reinterpret_cast<const uint4*>(q + (size_t)t * p.ld_q + (row0 + v - t * c.G) * DH)
                                : make_uint4(0u, 0u, 0u, 0u);
            };
            if constexpr (E8) {
                // three e5m2 parts, a power of two per row (the C lanes of a row are neighbours), eight rows at a time
#pragma unroll 1
                for (int i0 = 0; i0 < NI; i0 += 8) {
                    uint4 x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = load(v0 + (i0 + i) * RS);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                        float y[8], most = 0.f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            y[2 * k] = bf_lo(u[k]);
                            y[2 * k + 1] = bf_hi(u[k]);
                            most = max3(most, fabsf(y[2 * k]), fabsf(y[2 * k + 1]));
                        }
#pragma unroll
                        for (int o = C / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                        // (an infinity makes the row NaN, as its scores would be)
                        const bool inf = most > 3.402823466e38f;
                        const int e = inf ? 0 : query_exponent(most);
                        const float f = inf ? NAN : exp2_int(-e);
                        const int v = v0 + (i0 + i) * RS;
                        if (ch == 0) row_scale[begun & 1][w][v] = (int8_t)e;
                        unsigned char* d = q_s + w * kTile + v * DH + (((ch >> 1) ^ (DH == 128 ? v & 7 : v >> 1 & 3)) << 4) + (ch & 1) * 8;
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] *= f;
#pragma unroll
                        for (int part = 0; part < 3; ++part) {
                            uint32_t a[2];
#pragma unroll
                            for (int k = 0; k < 8; k += 4) {
                                a[k / 4] = encode4_e5m2(y[k], y[k + 1], y[k + 2], y[k + 3]);
                                if (part == 2) continue;
                                const float2 lo = decode2_e5m2((uint16_t)a[k / 4]), hi = decode2_e5m2((uint16_t)(a[k / 4] >> 16));
                                y[k] -= lo.x;
                                y[k + 1] -= lo.y;
                                y[k + 2] -= hi.x;
                                y[k + 3] -= hi.y;
                            }
                            *reinterpret_cast<uint2*>(d + part * 128 * DH) = make_uint2(a[0], a[1]);
                        }
                    }
                }
                ++begun;
            } else {
                uint4 x[NI];
#pragma unroll
                for (int i = 0; i < NI; ++i) x[i] = load(v0 + i * RS);
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int v = v0 + i * RS;
                    *reinterpret_cast<uint4*>(q_s + w * kTile + (ch >> 3) * kAtHalf + v * 128 + (((ch & 7) ^ (v & 7)) << 4)) = x[i];
                }
            }
            fence_proxy_async();  // the generic stores above, before the MMAs read them
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full + w);
            // the item after: its queries on their way into L2
            ItemWalk nx = it;
            nx.next(c, shape);
            if (nx.more() && nx.tokens(shape) * c.G > row0 + wt) {
                const int t = div_g(row0 + wt, g_magic);
                const bf16_t* r = static_cast<const bf16_t*>(p.q) + (size_t)(nx.q0 + nx.tile * shape.TP + t) * p.ld_q +
                                  (size_t)(nx.g * c.G + row0 + wt - t * c.G) * DH;
                asm volatile("prefetch.global.L2 [%0];" ::"l"(r));
                if (DH == 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(r + 64));
            }
        };
        if (wt == 0 && row0 == 0) reinterpret_cast<SharedItem*>(p.scratch)[me] = {0, 0, 0, -1};
        int sn = 0;  // pages seen
        bool ok = true;
        queries();
        while (it.more() && ok) {
            const int rows = min(128, it.tokens(shape) * c.G - row0), i0 = it.tile * shape.TP;
            const bool live = quad * 32 < rows;  // this warp has rows at all
            const int row = row0 + min(r, rows - 1), tr = div_g(row, g_magic), tok = i0 + tr;
            int pos = it.len - it.n + tok, lo = p.window > 0 ? pos - p.window + 1 : 0;
            if (shape.n_top > 0) {  // positions in the list's own order
                const int kept = pos < 0 ? 0 : min(shape.n_top, pos / kPage + 1);
                const int32_t* list = p.pages + ((size_t)(it.q0 + tok) * c.n_kv + it.g) * shape.n_top;
                if (kept > 0) pos = (kept - 1) * kPage + (list[kept - 1] == pos / kPage ? pos % kPage : kPage - 1);
            }
            float m_ref = E8 ? kNoScore : -INFINITY, l = 0.f;
            // 8-bit pools (codes.cuh): the reference is m_ref + v_ref; large: of m_ref; v_top: the largest scale so far
            float v_ref = 0.f, v_top = kNoScale;
            bool large = false;
            float c_row = c2;        // what the row's raw scores are worth
            if (E8) {
                ok = wait(q_full + w, (uint32_t)((begun - 1) & 1), 60, begun);
                if (!ok) break;
                c_row = c2 * exp2_int(row_scale[(begun - 1) & 1][w][r]);
            }
            // 8-bit pools: lane l holds the scales of page l of 32, those of the next 32 are on their way: blocks first,
            // scales eight pages later, so that no page waits for them
            const int pg0 = (it.t0 + it.kv0) * 2, gone = E8 ? first_seen(shape, it.n, it.len, it.tile) / kPage : 0;
            int next_blk = -1;
            float k_sc = 1.f, v_sc = 0.f, next_k = 1.f, next_v = 0.f;  // (values': logarithms)
            auto block_at = [&](int j) {  // (-1: gone, masked)
                const int i = pg0 + j + lane;
                return j + lane < it.pages() && i * kPage < it.len && i >= gone ? page_block(c, it.b, i) : -1;
            };
            auto scales_at = [&](int blk) {
                next_k = 1.f;
                next_v = 0.f;
                if (blk >= 0) {
                    next_k = p.k_scale[(size_t)blk * c.n_kv + it.g];
                    next_v = log2_scale(p.v_scale[(size_t)blk * c.n_kv + it.g]);
                }
            };
            if (E8) scales_at(block_at(0));
            // whole tiles over selected pages: this row's bits, 32 pages at a time
            const uint32_t* bits =
                SEL ? p.bits + ((size_t)(it.q0 + tok) * c.n_kv + it.g) * bit_words(c.max_pages) : nullptr;
            uint32_t word = 0;
            const int np = it.pages();
            for (int j = 0; j < np; ++j, ++sn) {
                const uint32_t s_buf = s_col + (uint32_t)((sn & 1) * 64);
                float cs = c2;
                float v_now = 0.f;
                if (E8) {
                    if ((j & 31) == 0) {
                        k_sc = next_k;
                        v_sc = next_v;
                        next_blk = block_at(j + 32);
                    } else if ((j & 31) == 8) {
                        scales_at(next_blk);
                    }
                    // (never 0: masked scores are -infinity)
                    cs = fmaxf(c_row * __shfl_sync(0xffffffffu, k_sc, j & 31), 1.17549435e-38f);
                    v_now = __shfl_sync(0xffffffffu, v_sc, j & 31);
                }
                ok = wait(&s_full[w][sn & 1], (uint32_t)((sn >> 1) & 1), 58, sn);
                if (!ok) break;
                tc_fence_after();
                bool sel = true;
                if (SEL) {
                    const int pg = (it.t0 + it.kv0) * 2 + j;
                    if (j == 0 || (pg & 31) == 0) word = bits[pg >> 5];
                    sel = word >> (pg & 31) & 1;
                }
                if (SEL && live && !__any_sync(0xffffffffu, sel)) {  // nobody's page: no weight on it
                    uint32_t none[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) none[i] = 0u;
                    tmem_st32(s_buf, none);
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                } else if (live) {
                    uint32_t s[2][32];
#pragma unroll
                    for (int i = 0; i < 2; ++i) tmem_ld32_issue(s_buf + 32 * i, s[i]);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 2; ++i) pin32(s[i]);
                    const int e0 = (it.t0 + it.kv0) * kTileEnt + j * kPage;
                    if (e0 + kPage - 1 > pos || e0 < lo) {
#pragma unroll
                        for (int i = 0; i < kPage; ++i)
                            if (e0 + i > pos || e0 + i < lo) s[i >> 5][i & 31] = 0xff800000u;
                    }
                    const float top = SEL && !sel ? -INFINITY : fmaxf(max32(s[0]), max32(s[1])) * cs;
                    // the reference moves when the maximum (8-bit pools: with the page's scale) has passed it by the slack,
                    // or it is the first one
                    const float v_up = v_now + kWeightUp;
                    float neg = E8 ? v_up - (m_ref + v_ref) : 0.f;
                    const bool move = E8 ? top + neg > kWeightTop : top > m_ref + kAtSlack;
                    const bool far = E8 && v_now < v_top - kFarScale;  // (the same for the warp)
                    float down = -v_up;                                // from weights to the sum's, as an exponent
                    v_top = fmaxf(v_top, v_now);
                    bool dead = false;
                    if (__any_sync(0xffffffffu, E8 ? move || large || far : move)) {
                        float f = 1.f;
                        bool scaled = true;
                        if (!E8) {
                            if (move) f = m_ref == -INFINITY ? 0.f : ex2(m_ref - top);
                            if (move) m_ref = top;
                            l *= f;
                        } else {
                            // (exact beside large scores too)
                            const float by = (m_ref - top) + (v_ref - v_now);
                            const bool move = by < -kAtSlack;
                            if (move) {
                                l = times_ex2(l, by);
                                f = ex2(by);
                                m_ref = top;
                                v_ref = v_now;
                                large = fabsf(m_ref) > kLargeScore;
                            }
                            neg = v_up - (m_ref + v_ref);
                            scaled = __any_sync(0xffffffffu, move);
                            const bool any_large = __any_sync(0xffffffffu, large);
                            if (any_large) {
#pragma unroll
                                for (int i = 0; i < kPage; ++i)
                                    s[i >> 5][i & 31] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(s[i >> 5][i & 31]), cs), m_ref));
                                cs = 1.f;
                                neg = v_up - v_ref;
                            }
                            if (far) {  // (relative to the page's own largest score; fp16 would have 0 for the weights)
                                const float up = (any_large ? top - m_ref : top) + neg;
                                dead = up < -40.f && top > -INFINITY;
                                if (dead) {
                                    neg -= up;
                                    down = up - v_up;
                                }
                            }
                        }
                        if (j > 0 && scaled) {  // the output so far, once the values of the page before are in it
                            ok = wait(&o_full[w][(sn - 1) & 1], (uint32_t)(((sn - 1) >> 1) & 1), 59, sn);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int h = 0; h < DH / 32; ++h) {
                                uint32_t o[32];
                                tmem_ld32_issue(o_col + 32 * h, o);
                                tmem_ld_wait();
                                pin32(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_st32(o_col + 32 * h, o);
                            }
                        }
                    }
                    // (a page that the row has not selected: exponents of -infinity)
                    if (!E8) neg = SEL && !sel ? -INFINITY : m_ref == -INFINITY ? 0.f : -m_ref;
                    // two columns at a time (paired fp32 instructions)
                    const uint64_t c22 = f32x2(cs, cs), neg2 = f32x2(neg, neg);
                    uint64_t sum[2] = {0ull, 0ull};
                    uint32_t pk[32], pl[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const uint64_t e = fma_f32x2(u32x2(s[i >> 4][2 * (i & 15)], s[i >> 4][2 * (i & 15) + 1]), c22, neg2);
                        const float p0 = ex2(__uint_as_float((uint32_t)e)), p1 = ex2(__uint_as_float((uint32_t)(e >> 32)));
                        sum[i & 1] = add_f32x2(sum[i & 1], f32x2(p0, p1));
                        pk[i] = E8 ? half2_of(p0, p1) : pack_bf16x2(p0, p1);
                        if (PARTS == 2) pl[i] = pack_bf16x2(p0 - bf_lo(pk[i]), p1 - bf_hi(pk[i]));
                    }
                    if (far) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) pk[i] = dead ? 0u : pk[i];
                    }
                    tmem_st32(s_buf, pk);
                    if (PARTS == 2) tmem_st32(s_buf + 32, pl);
                    sum[0] = add_f32x2(sum[0], sum[1]);
                    float part = __uint_as_float((uint32_t)sum[0]) + __uint_as_float((uint32_t)(sum[0] >> 32));
                    if (E8) part = far ? times_ex2(part, down) : part * ex2(down);
                    l += part;
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[w][sn & 1]);
            }
            if (!ok) break;
            // where this item's rows go
            const bool whole = it.whole();
            bf16_t* out = static_cast<bf16_t*>(p.out) + (size_t)(it.q0 + tok) * p.ld_out + (size_t)(it.g * c.G + row - tr * c.G) * DH;
            float* part = reinterpret_cast<float*>(p.scratch + part_off) +
                          ((size_t)me * 2 + (it.kv0 == 0 ? 1 : 0)) * part_floats(part_rows, DH);
            if (it.begun() && row0 + r == 0)
                reinterpret_cast<SharedItem*>(p.scratch)[me] = {it.q0 + i0, it.tokens(shape) * c.G, it.g,
                                                                it.last_worker(pieces[PAIR ? 0 : w])};
            // the scores of this item are all done: the next one's queries, whose first scores then run
            // under the values and the output below
            it.next(c, shape);
            queries();
            ok = wait(&o_full[w][(sn - 1) & 1], (uint32_t)(((sn - 1) >> 1) & 1), 59, sn);
            if (!ok) break;
            tc_fence_after();
            if (live) {
                // (8-bit pools: weights are held up, and parts are left as codes.cuh says)
                const float inv = l > 0.f ? (E8 ? 1.f / (1 << (int)kWeightUp) : 1.f) / l : 0.f;
                const PartRef ref = E8 && !whole ? part_ref(m_ref, v_ref, l) : PartRef{m_ref, l, 1.f};
#pragma unroll
                for (int h = 0; h < DH / 32; ++h) {
                    uint32_t v[32];
                    tmem_ld32_issue(o_col + 32 * h, v);
                    tmem_ld_wait();
                    pin32(v);
                    if (E8 && !whole) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * ref.by);
                    }
                    if (r < rows && whole) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            uint32_t x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                x[e] = pack_bf16x2(__uint_as_float(v[i + 2 * e]) * inv, __uint_as_float(v[i + 2 * e + 1]) * inv);
                            *reinterpret_cast<uint4*>(out + 32 * h + i) = make_uint4(x[0], x[1], x[2], x[3]);
                        }
                    } else if (r < rows) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)  // (four dims of all rows lie side by side)
                            *reinterpret_cast<uint4*>(part + ((size_t)(8 * h + i / 4) * part_rows + row0 + r) * 4) =
                                make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                    }
                    __syncwarp();
                }
                if (!whole && r < rows)
                    *reinterpret_cast<float2*>(part + (size_t)part_rows * DH + 2 * (row0 + r)) = make_float2(ref.m, ref.l);
            }
            tc_fence_before();  // the output is read, before the next item's values overwrite it
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace pipo
