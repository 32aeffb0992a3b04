// Block tables, lengths and slots of a step, from the requests' lengths.
//
// For request b, with H_b pages held, kept entries n_b (clamped to what is held) and a_b
// new tokens: pages from k_b = ceil(n_b / 64) on go back onto the stack of free
// blocks, request by request; w_b = ceil((n_b + a_b) / 64) - k_b pages are wanted.  b is served if its row
// has room, and if the stack holds the wanted pages of all requests up to b, and the
// token arrays their tokens (b with w_b = 0 needs only the latter).  The pages of all served
// requests are the last ones of the stack, in their order; so the same call on its own result
// changes nothing (unless kept entries were clamped: what is held has grown).
//
// Bound by latency: three prefix sums over the requests in one CTA (every request has its
// sums in shared memory), then a thread per page given back, per page taken and
// per token, each finding its request by bisection.
#pragma once

#include "paged.cuh"

namespace pipo {

constexpr int kTabThreads = 1024, kTabPer = kPagedMaxBatch / kTabThreads;  // requests of a thread
// Tokens up to which the same launch writes the slots too (16 requests, in a graph: 2048 tokens 6.8 us by one launch,
// 7.7 by two; 4096 7.6 and 7.8; 8192 9.5 and 7.9)
constexpr int kTabInline = 4096;

__host__ __device__ constexpr size_t tables_smem(int batch) { return (size_t)(4 * batch + 3) * 4; }

// inclusive sums of N values over the block's threads, and the totals
template <int N>
__device__ __forceinline__ void block_sums(long long (&x)[N], long long (&total)[N]) {
    __shared__ long long part[N][kTabThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const long long v = __shfl_up_sync(0xffffffffu, x[k], o);
            if (lane >= o) x[k] += v;
        }
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < N; ++k) part[k][warp] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        long long v = part[k][lane], before = lane < warp ? v : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            v += __shfl_xor_sync(0xffffffffu, v, o);
            before += __shfl_xor_sync(0xffffffffu, before, o);
        }
        x[k] += before;
        total[k] = v;
    }
}

// the last b with first[b] <= i (first[0] = 0; equal ones in a row: the last of them)
__device__ __forceinline__ int owner(const int* first, int batch, int i) {
    int lo = 0, hi = batch - 1;
    while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if (first[m] <= i) lo = m; else hi = m - 1;
    }
    return lo;
}

// slot and position of token t, from the finished tables
__device__ __forceinline__ void write_slot(const TablesArgs& p, const int* q_start, int t, int tokens, int keep_of_b, int b) {
    int pos = -1, slot = -1;
    if (t < tokens) {
        pos = keep_of_b + t - q_start[b];
        slot = p.table[(size_t)b * p.max_pages + pos / kPage] * kPage + pos % kPage;
    }
    p.slots[t] = slot;
    p.positions[t] = pos;
}

__global__ void __launch_bounds__(kTabThreads) page_tables_kernel(TablesArgs p) {
    extern __shared__ int tab_smem[];
    int* first_page = tab_smem;              // [batch] the first page given back or taken
    int* back = first_page + p.batch;        // [batch] pages given back by the requests before
    int* taken = back + p.batch;             // [batch] pages taken by them
    int* row = taken + p.batch;              // [batch + 1] tokens of them
    pdl_launch();
    pdl_wait();
    const int per = (p.batch + kTabThreads - 1) / kTabThreads, b0 = (int)threadIdx.x * per;
    const int n_free = min(max(*p.n_free, 0), p.n_blocks);
    int keep[kTabPer], k0[kTabPer], held[kTabPer], add[kTabPer];
    long long want[kTabPer];
    long long sum[3] = {0, 0, 0}, all[3];  // given back, wanted, asked tokens
#pragma unroll
    for (int i = 0; i < kTabPer; ++i) {
        const int b = b0 + i;
        const bool live = i < per && b < p.batch;
        held[i] = live ? min(max(p.held[b], 0), p.max_pages) : 0;
        keep[i] = live ? (int)min((long long)max(p.kept[b], 0), (long long)held[i] * kPage) : 0;
        add[i] = live ? max(p.added[b], 0) : 0;
        k0[i] = (keep[i] + kPage - 1) / kPage;
        want[i] = ((long long)keep[i] + add[i] + kPage - 1) / kPage - k0[i];
        if (k0[i] + want[i] > p.max_pages) want[i] = -1;  // no room in its row
        sum[0] += held[i] - k0[i];
        if (want[i] >= 0) {
            sum[1] += want[i];
            sum[2] += add[i];
        }
    }
    long long mine[3] = {sum[0], sum[1], sum[2]};
    block_sums<3>(sum, all);
#pragma unroll
    for (int k = 0; k < 3; ++k) sum[k] -= mine[k];
    const long long top = min((long long)n_free + all[0], (long long)p.n_blocks);
    long long got[2] = {0, 0}, total[2];  // pages taken, tokens
#pragma unroll
    for (int i = 0; i < kTabPer; ++i) {
        const int b = b0 + i;
        if (i < per && b < p.batch) {
            first_page[b] = k0[i];
            back[b] = (int)min(sum[0], (long long)p.n_blocks);
        }
        sum[0] += held[i] - k0[i];
        bool ok = want[i] >= 0;
        if (ok) {
            sum[1] += want[i];
            sum[2] += add[i];
            ok = (want[i] == 0 || sum[1] <= top) && sum[2] <= p.n_tokens;
        }
        if (!ok) want[i] = add[i] = 0;
        got[0] += want[i];
        got[1] += add[i];
    }
    long long own[2] = {got[0], got[1]};
    __syncthreads();  // (the sums' shared memory is used again)
    block_sums<2>(got, total);
#pragma unroll
    for (int k = 0; k < 2; ++k) got[k] -= own[k];
    const int n_back = (int)min(all[0], (long long)p.n_blocks), n_take = (int)total[0], tokens = (int)total[1];
    const int left = (int)top - n_take;
#pragma unroll
    for (int i = 0; i < kTabPer; ++i) {
        const int b = b0 + i;
        if (i >= per || b >= p.batch) continue;
        taken[b] = (int)got[0];
        row[b] = (int)got[1];
        p.q_start[b] = (int)got[1];
        p.kv_len[b] = keep[i] + add[i];
        p.held[b] = k0[i] + (int)want[i];
        got[0] += want[i];
        got[1] += add[i];
    }
    if (threadIdx.x == 0) {
        p.q_start[p.batch] = tokens;
        *p.n_free = left;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_back; i += kTabThreads) {
        const int b = owner(back, p.batch, i), page = first_page[b] + i - back[b];
        if (page >= p.max_pages) continue;  // (a state that holds more pages than there are blocks)
        int32_t* e = p.table + (size_t)b * p.max_pages + page;
        if (n_free + i < p.n_blocks) p.free_blocks[n_free + i] = *e;
        *e = -1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_take; i += kTabThreads) {
        const int b = owner(taken, p.batch, i);
        p.table[(size_t)b * p.max_pages + first_page[b] + i - taken[b]] = p.free_blocks[left + i];
    }
    if (p.n_tokens > kTabInline) return;
    __syncthreads();
    for (int t = threadIdx.x; t < p.n_tokens; t += kTabThreads) {
        const int b = t < tokens ? owner(row, p.batch, t) : 0;
        const int n = t < tokens ? (b + 1 < p.batch ? row[b + 1] : tokens) - row[b] : 0;
        write_slot(p, row, t, tokens, t < tokens ? p.kv_len[b] - n : 0, b);
    }
}

// the slots of many tokens, a thread each
__global__ void __launch_bounds__(256) page_slots_kernel(TablesArgs p) {
    pdl_launch();
    pdl_wait();
    const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
    if (t >= p.n_tokens) return;
    const int tokens = p.q_start[p.batch];
    const int b = t < tokens ? owner(p.q_start, p.batch, (int)t) : 0;
    const int keep = t < tokens ? p.kv_len[b] - (p.q_start[b + 1] - p.q_start[b]) : 0;
    write_slot(p, p.q_start, (int)t, tokens, keep, b);
}

}  // namespace pipo
