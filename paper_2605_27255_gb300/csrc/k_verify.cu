// Verification of drafted tokens: kernel and C entry point (a translation unit of its own).
#include <cstdio>

#include "pipo.h"
#include "verify.cuh"

namespace pipo {
void set_op_error(const char* msg);  // pipo_capi.cu: what pipo_last_error(NULL) returns on this thread

namespace {

template <typename T, int N>
cudaError_t verify_as(const VerifyArgs& a, cudaStream_t s) {
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3((unsigned)a.batch * kVerCluster);
    lc.blockDim = dim3(kVerThreads);
    lc.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, &verify_kernel<T, N>, a);
}

// Rows are read 16 bytes at a time where they all start on 16 bytes, else value by value
template <typename T>
cudaError_t verify_in(const VerifyArgs& a, cudaStream_t s) {
    constexpr int N = 16 / sizeof(T);
    const bool wide = reinterpret_cast<uintptr_t>(a.target) % 16 == 0 && a.ld_target % N == 0 &&
                      (!a.draft || (reinterpret_cast<uintptr_t>(a.draft) % 16 == 0 && a.ld_draft % N == 0));
    return wide ? verify_as<T, N>(a, s) : verify_as<T, 1>(a, s);
}

}  // namespace
}  // namespace pipo

using namespace pipo;

extern "C" pipo_status pipo_op_verify_drafts(int32_t dtype, int32_t vocab, int32_t batch, int32_t n_drafted,
                                             const void* d_target, int64_t ld_target, const void* d_draft, int64_t ld_draft,
                                             const int32_t* d_drafted, const int32_t* d_start, const float* d_u,
                                             const float* d_r, int32_t width, int32_t* d_tokens, int32_t* d_count,
                                             void* stream) {
    auto bad = [](const char* what) {
        char buf[160];
        snprintf(buf, sizeof buf, "pipo_op_verify_drafts: %s", what);
        set_op_error(buf);
        return PIPO_EINVAL;
    };
    if ((dtype != 0 && dtype != 1) || vocab < 1 || vocab > kVerMaxVocab || batch < 0 || batch > 65536 || n_drafted < 0 ||
        n_drafted > (1 << 30) || width < 1 || width > (1 << 20))
        return bad("bad type or sizes");
    if (batch == 0) return PIPO_OK;
    const uintptr_t es = dtype ? 2 : 4;
    auto rows = [&](const void* p, int64_t ld) {
        return p && reinterpret_cast<uintptr_t>(p) % es == 0 && ld >= vocab && ld <= (int64_t)1 << 40;
    };
    auto words = [](const void* p) { return p && reinterpret_cast<uintptr_t>(p) % 4 == 0; };
    if (!rows(d_target, ld_target) || !words(d_start) || !words(d_r) || !words(d_tokens) || !words(d_count) ||
        (n_drafted > 0 && (!words(d_drafted) || !words(d_u) || (d_draft && !rows(d_draft, ld_draft)))))
        return bad("bad arguments");
    VerifyArgs a{};
    a.target = d_target;
    a.draft = n_drafted > 0 ? d_draft : nullptr;
    a.ld_target = ld_target;
    a.ld_draft = ld_draft;
    a.drafted = d_drafted;
    a.start = d_start;
    a.u = d_u;
    a.r = d_r;
    a.vocab = vocab;
    a.batch = batch;
    a.n_drafted = n_drafted;
    a.width = width;
    a.tokens = d_tokens;
    a.count = d_count;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype ? verify_in<__nv_bfloat16>(a, s) : verify_in<float>(a, s);
    if (e == cudaSuccess) return PIPO_OK;
    char buf[256];
    snprintf(buf, sizeof buf, "pipo_op_verify_drafts: %s", cudaGetErrorString(e));
    set_op_error(buf);
    return PIPO_ECUDA;
}
