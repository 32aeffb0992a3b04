// Paged-cache operators: what the host code (paged_capi.cu) and the kernel
// units share.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pipo {

constexpr int kPage = 64;            // entries per block
constexpr int kPagedMaxBatch = 4096;
constexpr int kPagedMaxGroup = 16;   // query heads per kv head
constexpr int kPagedMaxTop = 4096;

// the cache and the ragged batch of new tokens (pipo_paged)
struct PagedArgs {
    void *k, *v, *means;
    const int32_t *table, *q_start, *kv_len;
    int dtype, n_q, n_kv, G, dh;
    int n_blocks, max_pages, batch, n_tokens;
};

struct AppendArgs {
    PagedArgs c;
    const void *q, *kn, *vn;      // fp32 or bf16, token t at q + t * ld_q
    long long ld_q, ld_k, ld_v;
    const void *q_gain, *k_gain;  // [dh] in the pools' type, or nullptr
    const float* rope;            // [position][dh / 2][2], or nullptr
    float eps;
    int in_bf16;
    void* q_out;                  // [n_tokens][n_q * dh] or nullptr
};

struct AttnPagedArgs {
    PagedArgs c;
    const void* q;
    long long ld_q;
    void* out;
    long long ld_out;
    float scale;
    int window;             // 0: none
    const int32_t* pages;   // [token][n_kv][n_top] kept pages, ascending, -1 behind the last; nullptr: every page
    int n_top;
    const uint32_t* bits;   // [token][n_kv][bit_words(max_pages)] the same as bits, for whole tiles, in place of the list; or nullptr
    unsigned char* scratch;
};

struct ScoreArgs {
    PagedArgs c;
    const void* q;
    long long ld_q;
    float scale;
    float* scores;  // [token][n_kv][max_pages]
};

struct SelectArgs {
    PagedArgs c;
    const float* scores;
    int n_top, n_sink, n_local;
    int32_t* pages;
    uint32_t* bits;  // or nullptr
};

inline __host__ __device__ int bit_words(int max_pages) { return (max_pages + 31) / 32; }

// How an attention launch is laid out
struct AttnPlan {
    int dev;
    bool pair;          // bf16: two 128-row tiles per item share the copies
    int rt;             // fp32: rows of a tile / 16
    bool join;          // items may be shared between workers
    bool listed;        // selected pages: a token's own list; else whole tiles with bits
    int TP;             // tokens per row tile
    long long tiles;    // row tiles at most
    int ctas, workers;
    int part_rows;      // rows of a partial
    size_t part_off;    // partials in the scratch
    size_t bits_off;    // selected pages as bits
    size_t scratch;     // bytes in all
};

AttnPlan plan_attn(const PagedArgs& c, int n_top, int dev, int sms);  // k_paged_tc.cu

// k_paged_tc.cu
cudaError_t launch_attn_tile(const AttnPagedArgs& a, const AttnPlan& pl, const CUtensorMap& tk, const CUtensorMap& tv,
                             cudaStream_t s);
cudaError_t take_error_paged(unsigned* code, unsigned* info);

// k_paged.cu
cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t s);
cudaError_t launch_page_scores(const ScoreArgs& a, cudaStream_t s);
cudaError_t launch_page_select(const SelectArgs& a, cudaStream_t s);
cudaError_t launch_attn_f32(const AttnPagedArgs& a, const AttnPlan& pl, cudaStream_t s);

}  // namespace pipo
