// How the attention kernels share a ragged batch.
//
// The rows of a sequence (its new tokens times the query heads of one kv head)
// are cut into row tiles of TP tokens; a row tile with one kv head is an item, and
// an item is nt units, one per tile of kTileEnt cache entries that its rows
// see.  The units of all items lie on one line (row tiles in order, within a
// tile head by head), each item's behind kItemCost more that stand for its queries and
// outputs, and S workers (or as many as the line is long) cut the line into equal pieces: worker
// i takes what lies in [i W / S, (i + 1) W / S).  So every worker has the same to do
// whatever the lengths are, a long cache with few rows is split over all of
// them, and with many rows at most one item at each end of a worker's piece
// is shared.  Of a shared item each worker leaves the running output, maximum
// and sum of its part in the scratch; combine_kernel joins them in order, so the
// result depends on the lengths alone, not on who came first.
#pragma once

#include "paged.cuh"

namespace pipo {

constexpr int kTileEnt = 128;  // entries per unit (two pages)
// What an item costs beside its units, in units: about 6300 cycles from the last page of one to
// the second of the next in the bf16 kernel, against 3300 for a unit.  (Without it the workers of 16
// mixed sequences took 75000 to 143000 cycles, by their number of items.)  The fp32 kernel cuts
// its pieces by the same number; it was not measured there.
constexpr int kItemCost = 2;

// What a launch needs of an item's shape
struct ItemShape {
    int TP;         // tokens per row tile
    int window;     // 0: none
    int n_top;      // > 0: the entries are those of listed pages, and TP = 1
};

// Row tile j of a sequence with n new tokens and len entries
struct RowTile {
    int t0, nt;     // first unit (in kTileEnt entries from the start of the cache or of the list), units
    int np;         // pages of them: 2 nt, or one less
};
// The first entry that any row of it sees.  Those before may hold anything (pages that the window
// has passed may be gone): they are not read, or their values are cleared.
__device__ __forceinline__ int first_seen(const ItemShape& s, int n, int len, int j) {
    return s.window > 0 ? max(0, len - n + j * s.TP - s.window + 1) : 0;
}
__device__ __forceinline__ RowTile row_tile(const ItemShape& s, int n, int len, int j) {
    const int i0 = j * s.TP, i1 = min(n, i0 + s.TP);
    const int last = len - n + i1 - 1;
    if (s.n_top > 0) {
        const int kept = last < 0 ? 0 : min(s.n_top, last / kPage + 1);
        return {0, max(1, (kept + 1) / 2), max(1, kept)};
    }
    const int hi = max(0, last + 1), lo = min(hi, first_seen(s, n, len, j));
    const int t0 = lo / kTileEnt, np = max(1, (hi + kPage - 1) / kPage - 2 * t0);
    return {t0, (np + 1) / 2, np};
}

__device__ __forceinline__ int seq_new(const PagedArgs& c, int b) { return max(0, q_row(c, b + 1) - q_row(c, b)); }

// The scratch: one record per worker, then the parts.  A worker leaves at most one
// item that it has begun for others to go on with, its last one.
struct alignas(16) SharedItem {
    int token, rows;   // first token row, rows
    int g, last;       // kv head; the last worker that shares it (-1: there is no such item)
};

__host__ __device__ inline long long tiles_bound(int n_tokens, int batch, int TP) {
    const long long a = n_tokens, b = n_tokens / TP + (long long)batch;
    return a < b ? a : b;
}
__host__ __device__ inline size_t record_bytes(int workers) { return ((size_t)workers * sizeof(SharedItem) + 255) / 256 * 256; }
// floats of one partial: [DH / 4][rows][4] outputs (a warp whose lanes are rows writes and
// reads them side by side), then (maximum, sum) of every row; an even number of rows keeps
// every partial 16-byte aligned
__host__ __device__ inline size_t part_floats(int rows, int dh) { return (size_t)rows * (dh + 2); }

// A worker's piece: where it starts, and how many units it has.
struct Piece {
    int b, tile, g, kv;  // sequence, row tile in it, head, unit within the item
    int left;            // of the line, from that unit on (0: nothing to do)
    long long end, total;  // end of the piece, length of the line
    int workers;         // S, or as many as the line is long
};

// Ints of shared memory that find_pieces uses
__host__ __device__ constexpr int find_ints(int batch) { return 3 * batch + 1; }

// All threads of a block (NT of them): the piece of each of its NW workers
// (w0 .. w0 + NW - 1 of S), written to `out` in shared memory.  tmp: find_ints(batch)
// ints of shared memory.
template <int NT, int NW>
__device__ __forceinline__ void find_pieces(const PagedArgs& c, const ItemShape& s, int w0, int S, int* tmp, Piece* out) {
    __shared__ long long warp_units[NT / 32];
    __shared__ int warp_tiles[NT / 32];
    int* seq_tiles = tmp;            // [batch + 1] row tiles before every sequence
    int* seq_n = tmp + c.batch + 1;  // [batch] new tokens, entries
    int* seq_l = seq_n + c.batch;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int tiles = 0;
    for (int b0 = 0; b0 < c.batch; b0 += NT) {
        const int b = b0 + tid;
        int n = 0;
        if (b < c.batch) {
            const int nn = seq_new(c, b);
            seq_n[b] = nn;
            seq_l[b] = seq_len(c, b);
            n = (nn + s.TP - 1) / s.TP;
        }
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (b0 > 0) __syncthreads();  // (the sums of the round before are read)
        if (lane == 31) warp_tiles[warp] = incl;
        __syncthreads();
        int before = tiles;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) {
            const int v = warp_tiles[w];
            if (w < warp) before += v;
            tiles += v;
        }
        if (b < c.batch) seq_tiles[b] = before + incl - n;
    }
    // (offsets that decrease could count rows twice: never more tiles than the scratch has room for)
    tiles = (int)min((long long)tiles, tiles_bound(c.n_tokens, c.batch, s.TP));
    if (tid == 0) seq_tiles[c.batch] = tiles;
    if (tid < NW) out[tid].left = 0;
    __syncthreads();
    // this thread's run of row tiles and its units
    const int x0 = (int)((long long)tiles * tid / NT), x1 = (int)((long long)tiles * (tid + 1) / NT);
    int lo = 0, hi = c.batch - 1;  // the last b with seq_tiles[b] <= x0 (it holds x0: an empty sequence's start is its successor's)
    while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (seq_tiles[m] <= x0) lo = m; else hi = m - 1;
    }
    const int bfirst = lo;
    auto walk = [&](auto&& fn) {  // fn(b, tile, shape) -> stop
        int b = bfirst;
        for (int x = x0; x < x1; ++x) {
            while (x >= seq_tiles[b + 1]) ++b;
            if (fn(b, x - seq_tiles[b], row_tile(s, seq_n[b], seq_l[b], x - seq_tiles[b]))) return;
        }
    };
    long long mine = 0;
    walk([&](int, int, const RowTile& r) {
        mine += (long long)(r.nt + kItemCost) * c.n_kv;
        return false;
    });
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) warp_units[warp] = incl;
    __syncthreads();
    long long total = 0, before = incl - mine;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const long long v = warp_units[w];
        if (w < warp) before += v;
        total += v;
    }
    const int Sw = (int)min((long long)S, total);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w0 + w >= Sw) break;
        const long long u0 = (long long)(w0 + w) * total / Sw, u1 = (long long)(w0 + w + 1) * total / Sw;
        if (u0 >= before && u0 < before + mine) {
            long long at = before;
            walk([&](int b, int j, const RowTile& r) {
                const int len = r.nt + kItemCost;
                const long long n = (long long)len * c.n_kv;
                if (u0 >= at + n) {
                    at += n;
                    return false;
                }
                const int g = (int)((u0 - at) / len), off = (int)((u0 - at) % len) - kItemCost;
                // (a piece that starts before the item's first unit)
                out[w] = {b, j, g, max(0, off), max(0, (int)(u1 - u0) + min(0, off)), u1, total, Sw};
                return true;
            });
        }
    }
    __syncthreads();
}

// the worker that holds place u of the line
__device__ __forceinline__ int worker_of(long long u, long long total, int S) { return (int)(((u + 1) * S - 1) / total); }

// One worker's items in turn.  Every thread of a role keeps its own; what is only
// asked of an item that starts here stays in the piece (shared memory).
struct ItemWalk {
    int b, tile, g, left;
    // the present item
    int n, len, q0;      // new tokens and entries of the sequence, row of its first new token
    int t0, nt, np;      // first unit, units and pages of the item
    int kv0, kv1;        // this worker's units of it
    __device__ __forceinline__ void start(const PagedArgs& c, const ItemShape& s, const Piece& p) {
        b = p.b;
        tile = p.tile;
        g = p.g;
        left = p.left;
        kv0 = p.kv;
        if (left > 0) load(c, s);
    }
    __device__ __forceinline__ void load(const PagedArgs& c, const ItemShape& s) {
        n = seq_new(c, b);
        len = seq_len(c, b);
        q0 = q_row(c, b);
        shape(s);
    }
    __device__ __forceinline__ void shape(const ItemShape& s) {
        const RowTile r = row_tile(s, n, len, tile);
        t0 = r.t0;
        nt = r.nt;
        np = r.np;
        kv1 = min(nt, kv0 + left);
    }
    __device__ __forceinline__ int pages() const { return min(2 * kv1, np) - 2 * kv0; }  // this worker's
    __device__ __forceinline__ bool more() const { return left > 0; }
    __device__ __forceinline__ bool whole() const { return kv0 == 0 && kv1 == nt; }
    __device__ __forceinline__ bool begun() const { return kv0 == 0 && kv1 < nt; }  // here, and not finished
    __device__ __forceinline__ int tokens(const ItemShape& s) const { return min(s.TP, n - tile * s.TP); }
    __device__ __forceinline__ void next(const PagedArgs& c, const ItemShape& s) {
        left = max(0, left - (kv1 - kv0) - kItemCost);
        kv0 = 0;
        if (left == 0) return;
        if (++g < c.n_kv) {
            kv1 = min(nt, left);
            return;
        }
        g = 0;
        if (++tile * s.TP < n) {
            shape(s);
            return;
        }
        tile = 0;
        do ++b;
        while (b + 1 < c.batch && seq_new(c, b) == 0);
        load(c, s);
    }
    // the last worker that holds a unit of this item, asked by the one with its first unit
    __device__ __forceinline__ int last_worker(const Piece& p) const {
        return worker_of(p.end - left + nt - 1, p.total, p.workers);
    }
};

// Joins the parts of the shared items: out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.
// grid (workers, groups of 32 rows, DH / dims of a block), 128 threads: the item that worker x
// began and did not finish; its own part is its second slot, those of the workers after it their first.
// A block takes 32 dims of 32 rows in 2 slices of the parts (a thread: one row, 16 dims; most
// items of chunks are shared by two), or, where no tile has more than 4 rows, 16 dims in 8
// slices (a thread: 4 dims), so that a few parts' loads are all in flight at once; the slices are
// added up in order.  (One thread for all parts of a row: 12 us of the 59 of four decoding
// sequences of 15.5 K entries.)
template <int DH, typename T, int RP>
__device__ __forceinline__ void join_rows(const AttnPagedArgs& a, const SharedItem& m, const float* parts, int part_rows,
                                          float* tmp) {
    constexpr int PS = RP == 32 ? 2 : 8, NC = RP == 32 ? 4 : 1, V = NC * 4 + 2;  // slices; 4-dim groups; values passed on
    constexpr int CG = 128 / (RP * PS);                                          // threads of a row and slice
    const int t = threadIdx.x, rl = t % RP, row = blockIdx.y * 32 + rl, ps = t * PS / 128;
    const int first = blockIdx.x, n = m.last - first + 1, c0 = (blockIdx.z * CG + t / RP % CG) * NC;
    const size_t step = part_floats(part_rows, DH);
    float M = -INFINITY, L = 0.f, o[NC][4] = {};
    if (row < m.rows) {
#pragma unroll 2
        for (int i = ps; i < n; i += PS) {
            const float* p = parts + ((size_t)(first + i) * 2 + (i == 0 ? 1 : 0)) * step;
            const float2 e = *reinterpret_cast<const float2*>(p + (size_t)part_rows * DH + 2 * row);
            float4 v[NC];
#pragma unroll
            for (int k = 0; k < NC; ++k) v[k] = *reinterpret_cast<const float4*>(p + ((size_t)(c0 + k) * part_rows + row) * 4);
            const float top = fmaxf(M, e.x), ref = top == -INFINITY ? 0.f : top, f = exp2f(M - ref), w = exp2f(e.x - ref);
            M = top;
            L = L * f + w * e.y;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                o[k][0] = fmaf(w, v[k].x, o[k][0] * f);
                o[k][1] = fmaf(w, v[k].y, o[k][1] * f);
                o[k][2] = fmaf(w, v[k].z, o[k][2] * f);
                o[k][3] = fmaf(w, v[k].w, o[k][3] * f);
            }
        }
    }
    constexpr int U = 128 / PS;  // threads of a slice
    if (ps > 0) {
        float* x = tmp + (size_t)(ps - 1) * U * V + t % U;
        x[0] = M;
        x[U] = L;
#pragma unroll
        for (int k = 0; k < NC * 4; ++k) x[(2 + k) * U] = o[k / 4][k % 4];
    }
    __syncthreads();
    if (ps > 0 || row >= m.rows) return;
#pragma unroll
    for (int q = 0; q < PS - 1; ++q) {
        const float* x = tmp + (size_t)q * U * V + t;
        const float mx = x[0], top = fmaxf(M, mx), ref = top == -INFINITY ? 0.f : top, f = exp2f(M - ref), w = exp2f(mx - ref);
        M = top;
        L = L * f + w * x[U];
#pragma unroll
        for (int k = 0; k < NC * 4; ++k) o[k / 4][k % 4] = fmaf(w, x[(2 + k) * U], o[k / 4][k % 4] * f);
    }
    const float inv = L > 0.f ? 1.0f / L : 0.f;
    const int G = a.c.G, tok = row / G;
    T* out = static_cast<T*>(a.out) + (size_t)(m.token + tok) * a.ld_out + (size_t)(m.g * G + row - tok * G) * DH + c0 * 4;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][e] *= inv;
        store_f<T, 4>(out + 4 * k, o[k]);
    }
}

template <int DH, typename T, int RP>
__global__ void __launch_bounds__(128) combine_kernel(AttnPagedArgs a, int workers, int part_rows, size_t part_off) {
    __shared__ float tmp[RP == 32 ? 64 * 18 : 7 * 16 * 6];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const SharedItem m = reinterpret_cast<const SharedItem*>(a.scratch)[blockIdx.x];
    const int left = m.rows - (int)blockIdx.y * 32;
    if (m.last <= (int)blockIdx.x || left <= 0) return;
    // (after a wait that gave up, the scratch may lack records: nothing outside it is read or written)
    if (m.last >= workers || m.rows > part_rows || m.g < 0 || m.g >= a.c.n_kv || m.token < 0 ||
        m.token + (m.rows - 1) / a.c.G >= a.c.n_tokens)
        return;
    const float* parts = reinterpret_cast<const float*>(a.scratch + part_off);
    join_rows<DH, T, RP>(a, m, parts, part_rows, tmp);
}

template <int DH, typename T>
inline cudaError_t launch_combine(const AttnPagedArgs& a, const AttnPlan& pl, cudaStream_t s) {
    if (!pl.join) return cudaSuccess;
    if (pl.part_rows <= 4)
        return launch_pdl(&combine_kernel<DH, T, 4>, dim3((unsigned)pl.workers, 1, DH / 16), 128, 0, s, a, pl.workers,
                          pl.part_rows, pl.part_off);
    return launch_pdl(&combine_kernel<DH, T, 32>, dim3((unsigned)pl.workers, (unsigned)((pl.part_rows + 31) / 32), DH / 32),
                      128, 0, s, a, pl.workers, pl.part_rows, pl.part_off);
}

}  // namespace pipo
