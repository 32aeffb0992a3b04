// Paged-cache operators: append, page scores, selection, attention on the CUDA
// cores (a translation unit of its own).
#include "append.cuh"
#include "attn_plain.cuh"
#include "select.cuh"

namespace pipo {

namespace {

unsigned ceil_div(long long a, long long b) { return (unsigned)((a + b - 1) / b); }

template <int DH, typename TI, typename T>
cudaError_t append_as(const AppendArgs& a, cudaStream_t s) {
    // pages that receive entries: a sequence with n new tokens spans at most n / 64 + 2
    const long long runs = a.c.n_tokens < a.c.n_tokens / kPage + 2LL * a.c.batch ? a.c.n_tokens
                                                                              : a.c.n_tokens / kPage + 2LL * a.c.batch;
    const int pages = (int)(runs * a.c.n_kv);
    const unsigned rows = a.q_out ? ceil_div((long long)a.c.n_tokens * a.c.n_q, kAppendWarps * kAppendRows) : 0;
    kv_append_kernel<DH, TI, T><<<pages + rows, kAppendWarps * 32, 0, s>>>(a, pages);
    return cudaGetLastError();
}

template <int DH, typename T>
cudaError_t append_in(const AppendArgs& a, cudaStream_t s) {
    return a.in_bf16 ? append_as<DH, bf16_t, T>(a, s) : append_as<DH, float, T>(a, s);
}

}  // namespace

cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t s) {
    if (a.c.dh == 64) return a.c.dtype ? append_in<64, bf16_t>(a, s) : append_in<64, float>(a, s);
    return a.c.dtype ? append_in<128, bf16_t>(a, s) : append_in<128, float>(a, s);
}

cudaError_t launch_page_scores(const ScoreArgs& a, cudaStream_t s) {
    const unsigned n = ceil_div((long long)a.c.n_tokens * a.c.n_kv, 4);
    if (a.c.dh == 64) {
        if (a.c.dtype) page_scores_kernel<64, bf16_t><<<n, 128, 0, s>>>(a);
        else page_scores_kernel<64, float><<<n, 128, 0, s>>>(a);
    } else {
        if (a.c.dtype) page_scores_kernel<128, bf16_t><<<n, 128, 0, s>>>(a);
        else page_scores_kernel<128, float><<<n, 128, 0, s>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t launch_page_select(const SelectArgs& a, cudaStream_t s) {
    page_select_kernel<<<ceil_div((long long)a.c.n_tokens * a.c.n_kv, 4), 128, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_attn_plain(const AttnPagedArgs& a, cudaStream_t s) {
    const unsigned n = ceil_div((long long)a.c.n_tokens * a.c.n_q, 4);
    if (a.c.dh == 64) {
        if (a.c.dtype) attn_plain_kernel<64, bf16_t><<<n, 128, 0, s>>>(a);
        else attn_plain_kernel<64, float><<<n, 128, 0, s>>>(a);
    } else {
        if (a.c.dtype) attn_plain_kernel<128, bf16_t><<<n, 128, 0, s>>>(a);
        else attn_plain_kernel<128, float><<<n, 128, 0, s>>>(a);
    }
    return cudaGetLastError();
}

}  // namespace pipo
