// Paged-cache operators: append, page scores, selection, attention on the CUDA
// cores (a translation unit of its own).
#include "append.cuh"
#include "attn_f32.cuh"
#include "select.cuh"

namespace pipo {

namespace {

unsigned ceil_div(long long a, long long b) { return (unsigned)((a + b - 1) / b); }

template <int DH, typename TI, typename T>
cudaError_t append_as(const AppendArgs& a, cudaStream_t s) {
    // pages that receive entries: a sequence with n new tokens spans at most n / 64 + 2
    const long long t = a.c.n_tokens, most = t / kPage + 2LL * a.c.batch, runs = t < most ? t : most;
    const int pages = (int)(runs * a.c.n_kv);
    const unsigned rows = a.q_out ? ceil_div(t, kAppendWarps) : 0;
    return launch_pdl(&kv_append_kernel<DH, TI, T>, dim3(pages + rows), kAppendWarps * 32, 0, s, a, pages);
}

template <int DH, typename T>
cudaError_t append_in(const AppendArgs& a, cudaStream_t s) {
    return a.in_bf16 ? append_as<DH, bf16_t, T>(a, s) : append_as<DH, float, T>(a, s);
}

template <int DH, typename T>
cudaError_t scores_as(const ScoreArgs& a, cudaStream_t s) {
    const unsigned y = ceil_div(a.c.max_pages, kScorePages);
    // Token by token below two tokens a sequence on average: a chunk's CTA costs about as much as
    // four single tokens', whose means are then read from L2 anyway.
    if ((long long)a.c.n_tokens < 2LL * a.c.batch || a.c.n_tokens < 4)
        return launch_pdl(&page_scores_kernel<DH, T>, dim3((unsigned)(a.c.n_tokens * (long long)a.c.n_kv), y), 128, 0, s, a);
    static thread_local int ready = -1;  // the shared-memory limit is set per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && ready != dev) {
        e = cudaFuncSetAttribute(&page_scores_chunk_kernel<DH, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)score_smem(DH));
        if (e == cudaSuccess) ready = dev;
    }
    if (e != cudaSuccess) return e;
    const long long t = a.c.n_tokens, most = t / kScoreTok + a.c.batch, tiles = t < most ? t : most;
    return launch_pdl(&page_scores_chunk_kernel<DH, T>, dim3((unsigned)(tiles * a.c.n_kv), y), 256, score_smem(DH), s, a);
}

template <int DH, int RT>
cudaError_t f32_as(const AttnPagedArgs& a, const AttnPlan& pl, cudaStream_t s) {
    auto* fn = &attn_f32_kernel<DH, RT>;
    static thread_local int ready = -1;  // the shared-memory limit is set per device
    if (ready != pl.dev) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)af_smem_for(DH, RT, kPagedMaxBatch));
        if (e != cudaSuccess) return e;
        ready = pl.dev;
    }
    const ItemShape shape{pl.TP, a.window, pl.listed ? a.n_top : 0};
    const cudaError_t e = launch_pdl(fn, dim3((unsigned)pl.ctas), kAfThreads, af_smem_for(DH, RT, a.c.batch), s, a, shape,
                                     pl.workers, pl.part_rows, pl.part_off);
    return e == cudaSuccess ? launch_combine<DH, float>(a, pl, s) : e;
}

}  // namespace

cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t s) {
    if (a.c.dh == 64) return a.c.dtype ? append_in<64, bf16_t>(a, s) : append_in<64, float>(a, s);
    return a.c.dtype ? append_in<128, bf16_t>(a, s) : append_in<128, float>(a, s);
}

cudaError_t launch_page_scores(const ScoreArgs& a, cudaStream_t s) {
    if (a.c.dh == 64) return a.c.dtype ? scores_as<64, bf16_t>(a, s) : scores_as<64, float>(a, s);
    return a.c.dtype ? scores_as<128, bf16_t>(a, s) : scores_as<128, float>(a, s);
}

cudaError_t launch_page_select(const SelectArgs& a, cudaStream_t s) {
    const dim3 n(ceil_div((long long)a.c.n_tokens * a.c.n_kv, 4));
    if (a.c.max_pages <= 128) return launch_pdl(&page_select_kernel<4>, n, 128, 0, s, a);
    if (a.c.max_pages <= 256) return launch_pdl(&page_select_kernel<8>, n, 128, 0, s, a);
    if (a.c.max_pages <= 1024) return launch_pdl(&page_select_kernel<32>, n, 128, 0, s, a);
    return launch_pdl(&page_select_kernel<0>, n, 128, 0, s, a);
}

cudaError_t launch_attn_f32(const AttnPagedArgs& a, const AttnPlan& pl, cudaStream_t s) {
    if (a.c.dh == 64) return pl.rt == 4 ? f32_as<64, 4>(a, pl, s) : f32_as<64, 1>(a, pl, s);
    return pl.rt == 4 ? f32_as<128, 4>(a, pl, s) : f32_as<128, 1>(a, pl, s);
}

}  // namespace pipo
