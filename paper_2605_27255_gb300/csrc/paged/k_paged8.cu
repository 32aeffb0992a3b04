// Operators on caches of e4m3 codes, and block tables (a translation unit of its own).
#include "append8.cuh"
#include "attn_few8.cuh"
#include "tables.cuh"

namespace pipo {

namespace {

unsigned ceil_div(long long a, long long b) { return (unsigned)((a + b - 1) / b); }

template <int DH>
cudaError_t append8_as(const AppendArgs& a, cudaStream_t s) {
    // pages that receive entries: a sequence with n new tokens spans at most n / 64 + 2
    const long long t = a.c.n_tokens, most = t / kPage + 2LL * a.c.batch, runs = t < most ? t : most;
    const int pages = (int)(runs * a.c.n_kv * 2);
    const dim3 grid(pages + (a.q_out ? ceil_div(t, kAppendWarps) : 0));
    return a.in_bf16 ? launch_pdl(&kv_append8_kernel<DH, bf16_t>, grid, kAppendWarps * 32, 0, s, a, pages)
                     : launch_pdl(&kv_append8_kernel<DH, float>, grid, kAppendWarps * 32, 0, s, a, pages);
}

template <int DH, int NT>
cudaError_t few8_as(const AttnPagedArgs& a, const AttnPlan& pl, cudaStream_t s) {
    auto* fn = &attn_few8_kernel<DH, NT>;
    static thread_local int ready = -1;  // the shared-memory limit is set per device
    if (ready != pl.dev) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)few_smem(DH, NT, kPagedMaxBatch));
        if (e != cudaSuccess) return e;
        ready = pl.dev;
    }
    const ItemShape shape{pl.TP, a.window, 0};
    const cudaError_t e = launch_pdl(fn, dim3((unsigned)pl.ctas), few_threads(DH, NT), few_smem(DH, NT, a.c.batch), s, a, shape,
                                     pl.workers, pl.part_rows, pl.part_off);
    // (blocks of 32 rows idle with tiles of 8.  Two builds in turn on one GPU: 16 sequences of 2000 entries and five rows 18.1
    // us with them, 16.5 so, eight of 15.5 K entries 48.6 and 47.6; 64 of five rows with a window of 1024 37.5 and 38.5)
    if (e == cudaSuccess && pl.join && NT == 1)
        return launch_pdl(&combine_kernel<DH, bf16_t, 8>, dim3((unsigned)pl.workers, 1, DH / 16), 128, 0, s, a, pl.workers,
                          pl.part_rows, pl.part_off);
    return e == cudaSuccess ? launch_combine<DH, bf16_t>(a, pl, s) : e;
}

}  // namespace

cudaError_t launch_kv_append8(const AppendArgs& a, cudaStream_t s) {
    return a.c.dh == 64 ? append8_as<64>(a, s) : append8_as<128>(a, s);
}

// The plan of attention over 8-bit pools by the rows (new tokens times query heads of a kv head) that the
// batch's sequences have on average: row tiles of 8, 16 or 32 rows on mma.sync; tiles of 128 on tcgen05, two
// pipelines with items of their own; above 128 rows pairs of tiles that share a pipeline's pages.  Where mma.sync
// would read the cache twice (33 to 64 rows) it goes by the work: with few sequences and heads its short start
// counts.  Measured in us, 32 query and 8 kv heads of 128 / 16 and 16 of 64, mma.sync, single tiles, pairs:
//   one sequence of 4000 entries, 64 rows   20 / 24    27 / 21    23 / 21
//   4 of 2000, 64 rows                      27 / 30    25 / 23    26 / 34
//   16 of 2000, 32 rows                     39 / 48    51 / 66    62 / 95
//   16 of 2000, 64 rows                     63 / 83    55 / 69    64 / 97
//   16 of 2000, 128 rows                   111 / 151   59 / 70    76 / 110
// (Uniform batches, no idle sequences: the average counts those too, so a chunk among many idle places takes tiles of
// few rows.)
constexpr int kFewRows = 32, kFewRowsStart = 64, kManyItems = 32;
AttnPlan plan_attn8(const PagedArgs& c, int dev, int sms) {
    AttnPlan pl{};
    pl.dev = dev;
    const long long mine = (long long)c.n_tokens * c.G;
    int per = 1;  // workers of an SM
    const int few = (long long)c.batch * c.n_kv >= kManyItems ? kFewRows : kFewRowsStart;
    if (mine > (long long)few * c.batch) {
        pl.pair = mine > 128LL * c.batch;
        pl.TP = (pl.pair ? 256 : 128) / c.G;
        per = pl.pair ? 1 : 2;
    } else {
        pl.rt = c.G <= 8 && mine <= 8LL * c.batch ? 1 : mine <= 16LL * c.batch ? 2 : 4;
        pl.TP = 8 * pl.rt / c.G;
        per = few_ctas(c.dh, pl.rt);
    }
    pl.tiles = tiles_bound(c.n_tokens, c.batch, pl.TP);
    const long long each = (c.max_pages + 1) / 2, most = pl.tiles * c.n_kv * each, all = (long long)sms * per;
    pl.workers = pl.ctas = (int)(most < all ? most : all);
    if (!pl.rt && !pl.pair) {  // two workers of a CTA
        pl.ctas = (pl.workers + 1) / 2;
        pl.workers = 2 * pl.ctas;
    }
    pl.join = each > 1;
    pl.part_rows = (int)(mine < (long long)pl.TP * c.G ? mine : (long long)pl.TP * c.G);
    pl.part_rows += pl.part_rows & 1;
    pl.part_off = record_bytes(pl.workers);
    pl.bits_off = pl.scratch = pl.part_off + (size_t)pl.workers * 2 * part_floats(pl.part_rows, c.dh) * sizeof(float);
    return pl;
}

cudaError_t launch_attn_few8(const AttnPagedArgs& a, const AttnPlan& pl, cudaStream_t s) {
    if (a.c.dh == 64) return pl.rt == 1 ? few8_as<64, 1>(a, pl, s) : pl.rt == 2 ? few8_as<64, 2>(a, pl, s) : few8_as<64, 4>(a, pl, s);
    return pl.rt == 1 ? few8_as<128, 1>(a, pl, s) : pl.rt == 2 ? few8_as<128, 2>(a, pl, s) : few8_as<128, 4>(a, pl, s);
}

cudaError_t launch_page_tables(const TablesArgs& a, cudaStream_t s) {
    static thread_local int ready = -1;  // the shared-memory limit is set per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && ready != dev) {
        e = cudaFuncSetAttribute(&page_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tables_smem(kPagedMaxBatch));
        if (e == cudaSuccess) ready = dev;
    }
    if (e == cudaSuccess) e = launch_pdl(&page_tables_kernel, dim3(1), kTabThreads, tables_smem(a.batch), s, a);
    if (e == cudaSuccess && a.n_tokens > kTabInline)
        e = launch_pdl(&page_slots_kernel, dim3(ceil_div(a.n_tokens, 256)), 256, 0, s, a);
    return e;
}

}  // namespace pipo
