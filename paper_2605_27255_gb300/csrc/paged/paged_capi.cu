// C entry points of the paged-cache operators: argument checks and launches.
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>

#include "paged.h"
#include "pipo.h"

namespace pipo {
void set_op_error(const char* msg);  // pipo_capi.cu: what pipo_last_error(NULL) returns on this thread
}

using namespace pipo;

namespace {

pipo_status fail(pipo_status s, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_op_error(buf);
    return s;
}

pipo_status cuda_status(const char* who, cudaError_t e) {
    return e == cudaSuccess ? PIPO_OK : fail(PIPO_ECUDA, "%s: %s", who, cudaGetErrorString(e));
}

bool a16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool a4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// the description's own fields (not the pools)
bool paged_ok(const pipo_paged* c, int32_t n_tokens) {
    return c && (c->dtype == 0 || c->dtype == 1) && c->n_kv_heads >= 1 && c->n_q_heads >= 1 &&
           c->n_q_heads % c->n_kv_heads == 0 && c->n_q_heads / c->n_kv_heads <= kPagedMaxGroup &&
           c->n_q_heads <= 65536 && (c->head_dim == 64 || c->head_dim == 128) && c->page_size == kPage &&
           c->n_blocks >= 1 && (long long)c->n_blocks * c->n_kv_heads * kPage <= 0x7fffffffLL && c->max_pages >= 1 &&
           c->max_pages <= 65535 * kPage && c->batch >= 0 && c->batch <= kPagedMaxBatch && n_tokens >= 0 &&
           (long long)n_tokens * c->n_q_heads <= (1 << 30);
}

bool batch_ok(const pipo_paged* c) {
    return c->table && c->q_start && c->kv_len && a4(c->table) && a4(c->q_start) && a4(c->kv_len);
}

bool pools_ok(const pipo_paged* c) { return c->k && c->v && a16(c->k) && a16(c->v); }

size_t esize(const pipo_paged* c) { return c->dtype ? 2 : 4; }

bool rows_ok(const void* p, int64_t ld, int64_t width, size_t es) {
    return p && a16(p) && ld >= width && ld <= (int64_t)1 << 40 && (ld * (int64_t)es) % 16 == 0;
}

PagedArgs args_of(const pipo_paged* c, int32_t n_tokens) {
    PagedArgs a{};
    a.k = c->k;
    a.v = c->v;
    a.means = c->means;
    a.table = c->table;
    a.q_start = c->q_start;
    a.kv_len = c->kv_len;
    a.dtype = c->dtype;
    a.n_q = c->n_q_heads;
    a.n_kv = c->n_kv_heads;
    a.G = c->n_q_heads / c->n_kv_heads;
    a.dh = c->head_dim;
    a.n_blocks = c->n_blocks;
    a.max_pages = c->max_pages;
    a.batch = c->batch;
    a.n_tokens = n_tokens;
    return a;
}

bool attn_args_ok(const pipo_paged* c, int32_t n_tokens, const void* d_q, int64_t ld_q, float scale, void* d_out,
                  int64_t ld_out) {
    const int64_t w = (int64_t)c->n_q_heads * c->head_dim;
    return batch_ok(c) && pools_ok(c) && rows_ok(d_q, ld_q, w, esize(c)) && rows_ok(d_out, ld_out, w, esize(c)) &&
           scale > 0.f && std::isfinite(scale);
}

// current device and its SMs
cudaError_t device_of(int* dev, int* sms) {
    static thread_local int have = -1, count = 0;
    cudaError_t e = cudaGetDevice(dev);
    if (e == cudaSuccess && have != *dev) {
        e = cudaDeviceGetAttribute(&count, cudaDevAttrMultiProcessorCount, *dev);
        if (e == cudaSuccess) have = *dev;
    }
    *sms = count;
    return e;
}

PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
std::mutex g_encode_lock;

// a pool as [n_blocks * n_kv * 64][d_h]: bf16 in boxes of one page x 64 dims, 128-byte swizzle; codes in
// boxes of one page, swizzled by the row's length (key codes) or as they lie there
enum class PoolKind { kBf16, kKeyCodes, kValueCodes };
pipo_status pool_map(const char* who, CUtensorMap* tm, void* pool, const PagedArgs& a, PoolKind kind = PoolKind::kBf16) {
    const bool codes = kind != PoolKind::kBf16;
    {
        std::lock_guard<std::mutex> lk(g_encode_lock);
        if (!g_encode) {
            void* fn = nullptr;
            cudaDriverEntryPointQueryResult q{};
            const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
            if (e != cudaSuccess) return cuda_status(who, e);
            if (q != cudaDriverEntryPointSuccess || !fn) return fail(PIPO_ECUDA, "%s: no cuTensorMapEncodeTiled", who);
            g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
        }
    }
    const cuuint64_t dims[2] = {(cuuint64_t)a.dh, (cuuint64_t)a.n_blocks * a.n_kv * kPage};
    const CUtensorMapSwizzle swizzle = kind == PoolKind::kValueCodes ? CU_TENSOR_MAP_SWIZZLE_NONE
                                       : codes && a.dh == 64         ? CU_TENSOR_MAP_SWIZZLE_64B
                                                                     : CU_TENSOR_MAP_SWIZZLE_128B;
    const cuuint64_t strides[1] = {(cuuint64_t)a.dh * (codes ? 1 : 2)};
    const cuuint32_t box[2] = {codes ? (cuuint32_t)a.dh : 64, (cuuint32_t)kPage}, es[2] = {1, 1};
    const CUresult r = g_encode(tm, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, pool, dims,
                                strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                swizzle,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? PIPO_OK : fail(PIPO_ECUDA, "%s: cuTensorMapEncodeTiled: error %d", who, (int)r);
}

// Scratch and launches of the attention calls; sel: the selection that comes first, or nullptr
pipo_status run_attn(const char* who, AttnPagedArgs a, SelectArgs* sel, size_t scratch_bytes, cudaStream_t s) {
    int dev = 0, sms = 0;
    cudaError_t e = device_of(&dev, &sms);
    if (e != cudaSuccess) return cuda_status(who, e);
    const AttnPlan pl = plan_attn(a.c, sel ? sel->n_top : 0, dev, sms);
    if (scratch_bytes < pl.scratch)
        return fail(PIPO_EINVAL, "%s: scratch needs %zu bytes, got %zu", who, pl.scratch, scratch_bytes);
    if (sel) {
        if (!pl.listed) a.bits = sel->bits = reinterpret_cast<uint32_t*>(a.scratch + pl.bits_off);
        e = launch_page_select(*sel, s);
        if (e != cudaSuccess) return cuda_status(who, e);
    }
    if (!a.c.dtype) return cuda_status(who, launch_attn_f32(a, pl, s));
    CUtensorMap tk, tv;
    pipo_status st = pool_map(who, &tk, a.c.k, a.c);
    if (st == PIPO_OK) st = pool_map(who, &tv, a.c.v, a.c);
    return st == PIPO_OK ? cuda_status(who, launch_attn_tile(a, pl, tk, tv, s)) : st;
}

// the checked arguments of an append
pipo_status append_args(const char* who, const pipo_paged* c, int32_t n_tokens, int32_t in_dtype, const void* d_q,
                        int64_t ld_q, const void* d_k, int64_t ld_k, const void* d_v, int64_t ld_v, const void* d_q_gain,
                        const void* d_k_gain, float eps, const float* d_rope, int32_t n_rope, void* d_q_out, AppendArgs* out) {
    const size_t es = in_dtype ? 2 : 4;
    const int64_t kd = (int64_t)c->n_kv_heads * c->head_dim;
    if (!batch_ok(c) || !pools_ok(c) || !rows_ok(d_k, ld_k, kd, es) || !rows_ok(d_v, ld_v, kd, es) ||
        (d_q != nullptr) != (d_q_out != nullptr) ||
        (d_q && (!rows_ok(d_q, ld_q, (int64_t)c->n_q_heads * c->head_dim, es) || !a16(d_q_out))) || !a16(c->means) ||
        !a16(d_q_gain) || !a16(d_k_gain) || !a16(d_rope) || !(eps >= 0.f) || !std::isfinite(eps))
        return fail(PIPO_EINVAL, "%s: bad arguments", who);
    if (d_rope && (int64_t)n_rope < (int64_t)kPage * c->max_pages)
        return fail(PIPO_EINVAL, "%s: %d rotations for %lld positions", who, n_rope, (long long)kPage * c->max_pages);
    AppendArgs a{};
    a.c = args_of(c, n_tokens);
    a.q = d_q;
    a.kn = d_k;
    a.vn = d_v;
    a.ld_q = ld_q;
    a.ld_k = ld_k;
    a.ld_v = ld_v;
    a.q_gain = d_q_gain;
    a.k_gain = d_k_gain;
    a.rope = d_rope;
    a.eps = eps;
    a.in_bf16 = in_dtype;
    a.q_out = d_q_out;
    *out = a;
    return PIPO_OK;
}

// an 8-bit cache as the other calls' description (the checks of sizes are theirs)
pipo_paged plain_of(const pipo_paged8* c) {
    pipo_paged x{};
    if (!c) return x;  // (page_size 0: refused)
    x.dtype = 1;
    x.n_q_heads = c->n_q_heads;
    x.n_kv_heads = c->n_kv_heads;
    x.head_dim = c->head_dim;
    x.page_size = c->page_size;
    x.n_blocks = c->n_blocks;
    x.max_pages = c->max_pages;
    x.batch = c->batch;
    x.k = c->k;
    x.v = c->v;
    x.table = c->table;
    x.q_start = c->q_start;
    x.kv_len = c->kv_len;
    return x;
}

bool scales_ok(const pipo_paged8* c) { return c->k_scale && c->v_scale && a4(c->k_scale) && a4(c->v_scale); }

}  // namespace

extern "C" {

pipo_status pipo_op_kv_append(const pipo_paged* c, int32_t n_tokens, int32_t in_dtype, const void* d_q, int64_t ld_q,
                              const void* d_k, int64_t ld_k, const void* d_v, int64_t ld_v, const void* d_q_gain,
                              const void* d_k_gain, float eps, const float* d_rope, int32_t n_rope, void* d_q_out,
                              void* stream) {
    if (!paged_ok(c, n_tokens) || (in_dtype != 0 && in_dtype != 1))
        return fail(PIPO_EINVAL, "pipo_op_kv_append: bad cache description or token count");
    if (c->batch == 0 || n_tokens == 0) return PIPO_OK;
    AppendArgs a{};
    const pipo_status st = append_args("pipo_op_kv_append", c, n_tokens, in_dtype, d_q, ld_q, d_k, ld_k, d_v, ld_v, d_q_gain,
                                       d_k_gain, eps, d_rope, n_rope, d_q_out, &a);
    if (st != PIPO_OK) return st;
    return cuda_status("pipo_op_kv_append", launch_kv_append(a, static_cast<cudaStream_t>(stream)));
}

size_t pipo_op_attn_paged_scratch(const pipo_paged* c, int32_t n_tokens) {
    int dev = 0, sms = 0;
    if (!paged_ok(c, n_tokens) || device_of(&dev, &sms) != cudaSuccess) return 0;
    if (c->batch == 0 || n_tokens == 0) return 16;
    const PagedArgs a = args_of(c, n_tokens);
    // every page (with the selection as bits, where tiles take it), or a token's own list
    const size_t bits = (size_t)n_tokens * c->n_kv_heads * bit_words(c->max_pages) * 4;
    return std::max(plan_attn(a, 0, dev, sms).scratch + bits, plan_attn(a, -1, dev, sms).scratch);
}

pipo_status pipo_op_attn_paged(const pipo_paged* c, int32_t n_tokens, const void* d_q, int64_t ld_q, float scale,
                               int32_t window, void* d_out, int64_t ld_out, void* d_scratch, size_t scratch_bytes,
                               void* stream) {
    if (!paged_ok(c, n_tokens) || window < 0)
        return fail(PIPO_EINVAL, "pipo_op_attn_paged: bad cache description, token count or window");
    if (c->batch == 0 || n_tokens == 0) return PIPO_OK;
    if (!attn_args_ok(c, n_tokens, d_q, ld_q, scale, d_out, ld_out) || !d_scratch || !a16(d_scratch))
        return fail(PIPO_EINVAL, "pipo_op_attn_paged: bad arguments");
    const size_t need = pipo_op_attn_paged_scratch(c, n_tokens);
    if (need == 0 || scratch_bytes < need)
        return fail(PIPO_EINVAL, "pipo_op_attn_paged: scratch needs %zu bytes, got %zu", need, scratch_bytes);
    AttnPagedArgs a{};
    a.c = args_of(c, n_tokens);
    a.q = d_q;
    a.ld_q = ld_q;
    a.out = d_out;
    a.ld_out = ld_out;
    a.scale = scale;
    // a window as long as any sequence is none; below that, positions minus the window fit in 32 bits
    a.window = (long long)window < (long long)kPage * c->max_pages ? window : 0;
    a.scratch = static_cast<unsigned char*>(d_scratch);
    return run_attn("pipo_op_attn_paged", a, nullptr, scratch_bytes, static_cast<cudaStream_t>(stream));
}

pipo_status pipo_op_page_scores(const pipo_paged* c, int32_t n_tokens, const void* d_q, int64_t ld_q, float scale,
                                float* d_scores, void* stream) {
    if (!paged_ok(c, n_tokens))
        return fail(PIPO_EINVAL, "pipo_op_page_scores: bad cache description or token count");
    if (c->batch == 0 || n_tokens == 0) return PIPO_OK;
    if (!batch_ok(c) || !c->means || !a16(c->means) ||
        !rows_ok(d_q, ld_q, (int64_t)c->n_q_heads * c->head_dim, esize(c)) || !(scale > 0.f) || !std::isfinite(scale) ||
        !d_scores || !a16(d_scores))
        return fail(PIPO_EINVAL, "pipo_op_page_scores: bad arguments");
    ScoreArgs a{};
    a.c = args_of(c, n_tokens);
    a.q = d_q;
    a.ld_q = ld_q;
    a.scale = scale;
    a.scores = d_scores;
    return cuda_status("pipo_op_page_scores", launch_page_scores(a, static_cast<cudaStream_t>(stream)));
}

pipo_status pipo_op_attn_pages(const pipo_paged* c, int32_t n_tokens, const void* d_q, int64_t ld_q, float scale,
                               const float* d_scores, int32_t n_top, int32_t n_sink, int32_t n_local, void* d_out,
                               int64_t ld_out, int32_t* d_pages, void* d_scratch, size_t scratch_bytes, void* stream) {
    if (!paged_ok(c, n_tokens) || n_top < 1 || n_top > kPagedMaxTop || n_sink < 0 || n_local < 0 || n_sink > n_top ||
        n_local > n_top - n_sink)
        return fail(PIPO_EINVAL, "pipo_op_attn_pages: bad cache description, token count or page counts");
    if (c->batch == 0 || n_tokens == 0) return PIPO_OK;
    if (!attn_args_ok(c, n_tokens, d_q, ld_q, scale, d_out, ld_out) || !d_scores || !a16(d_scores) || !d_pages ||
        !a16(d_pages) || !d_scratch || !a16(d_scratch))
        return fail(PIPO_EINVAL, "pipo_op_attn_pages: bad arguments");
    const size_t need = pipo_op_attn_paged_scratch(c, n_tokens);
    if (need == 0 || scratch_bytes < need)
        return fail(PIPO_EINVAL, "pipo_op_attn_pages: scratch needs %zu bytes, got %zu", need, scratch_bytes);
    SelectArgs sel{};
    sel.c = args_of(c, n_tokens);
    sel.scores = d_scores;
    sel.n_top = n_top;
    sel.n_sink = n_sink;
    sel.n_local = n_local;
    sel.pages = d_pages;
    AttnPagedArgs a{};
    a.c = sel.c;
    a.q = d_q;
    a.ld_q = ld_q;
    a.out = d_out;
    a.ld_out = ld_out;
    a.scale = scale;
    a.pages = d_pages;
    a.n_top = n_top;
    a.scratch = static_cast<unsigned char*>(d_scratch);
    return run_attn("pipo_op_attn_pages", a, &sel, scratch_bytes, static_cast<cudaStream_t>(stream));
}

pipo_status pipo_op_kv_append8(const pipo_paged8* c8, int32_t n_tokens, int32_t in_dtype, const void* d_q, int64_t ld_q,
                               const void* d_k, int64_t ld_k, const void* d_v, int64_t ld_v, const void* d_q_gain,
                               const void* d_k_gain, float eps, const float* d_rope, int32_t n_rope, void* d_q_out,
                               void* stream) {
    const pipo_paged desc = plain_of(c8), *c = &desc;
    if (!paged_ok(c, n_tokens) || (in_dtype != 0 && in_dtype != 1))
        return fail(PIPO_EINVAL, "pipo_op_kv_append8: bad cache description or token count");
    if (c->batch == 0 || n_tokens == 0) return PIPO_OK;
    AppendArgs a{};
    const pipo_status st = append_args("pipo_op_kv_append8", c, n_tokens, in_dtype, d_q, ld_q, d_k, ld_k, d_v, ld_v, d_q_gain,
                                       d_k_gain, eps, d_rope, n_rope, d_q_out, &a);
    if (st != PIPO_OK) return st;
    if (!scales_ok(c8)) return fail(PIPO_EINVAL, "pipo_op_kv_append8: bad scales");
    a.k_scale = c8->k_scale;
    a.v_scale = c8->v_scale;
    return cuda_status("pipo_op_kv_append8", launch_kv_append8(a, static_cast<cudaStream_t>(stream)));
}

size_t pipo_op_attn_paged8_scratch(const pipo_paged8* c8, int32_t n_tokens) {
    int dev = 0, sms = 0;
    const pipo_paged desc = plain_of(c8), *c = &desc;
    if (!paged_ok(c, n_tokens) || device_of(&dev, &sms) != cudaSuccess) return 0;
    if (c->batch == 0 || n_tokens == 0) return 16;
    return plan_attn8(args_of(c, n_tokens), dev, sms).scratch;
}

pipo_status pipo_op_attn_paged8(const pipo_paged8* c8, int32_t n_tokens, const void* d_q, int64_t ld_q, float scale,
                                int32_t window, void* d_out, int64_t ld_out, void* d_scratch, size_t scratch_bytes,
                                void* stream) {
    const pipo_paged desc = plain_of(c8), *c = &desc;
    if (!paged_ok(c, n_tokens) || window < 0)
        return fail(PIPO_EINVAL, "pipo_op_attn_paged8: bad cache description, token count or window");
    if (c->batch == 0 || n_tokens == 0) return PIPO_OK;
    if (!attn_args_ok(c, n_tokens, d_q, ld_q, scale, d_out, ld_out) || !scales_ok(c8) || !d_scratch || !a16(d_scratch))
        return fail(PIPO_EINVAL, "pipo_op_attn_paged8: bad arguments");
    int dev = 0, sms = 0;
    const cudaError_t e = device_of(&dev, &sms);
    if (e != cudaSuccess) return cuda_status("pipo_op_attn_paged8", e);
    AttnPagedArgs a{};
    a.c = args_of(c, n_tokens);
    const AttnPlan pl = plan_attn8(a.c, dev, sms);
    if (scratch_bytes < pl.scratch)
        return fail(PIPO_EINVAL, "pipo_op_attn_paged8: scratch needs %zu bytes, got %zu", pl.scratch, scratch_bytes);
    a.q = d_q;
    a.ld_q = ld_q;
    a.out = d_out;
    a.ld_out = ld_out;
    a.scale = scale;
    a.window = (long long)window < (long long)kPage * c->max_pages ? window : 0;
    a.scratch = static_cast<unsigned char*>(d_scratch);
    a.k_scale = c8->k_scale;
    a.v_scale = c8->v_scale;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (pl.rt) return cuda_status("pipo_op_attn_paged8", launch_attn_few8(a, pl, s));
    CUtensorMap tk, tv;
    pipo_status st = pool_map("pipo_op_attn_paged8", &tk, a.c.k, a.c, PoolKind::kKeyCodes);
    if (st == PIPO_OK) st = pool_map("pipo_op_attn_paged8", &tv, a.c.v, a.c, PoolKind::kValueCodes);
    return st == PIPO_OK ? cuda_status("pipo_op_attn_paged8", launch_attn_tile8(a, pl, tk, tv, s)) : st;
}

pipo_status pipo_op_page_tables(const pipo_page_tables* p, const int32_t* d_kept, const int32_t* d_added, int32_t n_tokens,
                                int32_t* d_q_start, int32_t* d_kv_len, int32_t* d_slots, int32_t* d_positions,
                                void* stream) {
    if (!p || p->batch < 0 || p->batch > kPagedMaxBatch || p->max_pages < 1 || p->max_pages > 65535 * kPage ||
        p->n_blocks < 1 || (long long)p->n_blocks * kPage > 0x7fffffffLL || n_tokens < 0 || n_tokens > (1 << 30))
        return fail(PIPO_EINVAL, "pipo_op_page_tables: bad sizes");
    if (p->batch == 0) return PIPO_OK;
    for (const void* x : {(const void*)p->table, (const void*)p->held, (const void*)p->free_blocks, (const void*)p->n_free,
                          (const void*)d_kept, (const void*)d_added, (const void*)d_q_start, (const void*)d_kv_len})
        if (!x || !a4(x)) return fail(PIPO_EINVAL, "pipo_op_page_tables: bad arguments");
    if (n_tokens > 0 && (!d_slots || !d_positions || !a4(d_slots) || !a4(d_positions)))
        return fail(PIPO_EINVAL, "pipo_op_page_tables: bad arguments");
    TablesArgs a{};
    a.table = p->table;
    a.held = p->held;
    a.free_blocks = p->free_blocks;
    a.n_free = p->n_free;
    a.kept = d_kept;
    a.added = d_added;
    a.max_pages = p->max_pages;
    a.n_blocks = p->n_blocks;
    a.batch = p->batch;
    a.n_tokens = n_tokens;
    a.q_start = d_q_start;
    a.kv_len = d_kv_len;
    a.slots = d_slots;
    a.positions = d_positions;
    return cuda_status("pipo_op_page_tables", launch_page_tables(a, static_cast<cudaStream_t>(stream)));
}

pipo_status pipo_op_paged_check(uint32_t* h_info) {
    cudaError_t e = cudaDeviceSynchronize();
    unsigned code = 0, info[4] = {0, 0, 0, 0};
    if (e == cudaSuccess) e = take_error_paged(&code, info);
    if (e != cudaSuccess) return cuda_status("pipo_op_paged_check", e);
    if (h_info)
        for (int i = 0; i < 4; ++i) h_info[i] = info[i];
    if (code)
        return fail(PIPO_ECUDA, "device wait timed out (code %u; first at wait site %u, block %u)", code, info[0],
                    info[1]);
    return PIPO_OK;
}

}  // extern "C"
