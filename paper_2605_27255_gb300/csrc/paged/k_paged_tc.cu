// Paged-cache attention on the tensor cores (a translation unit of its own).
#include "attn_f32.cuh"
#include "attn_tile.cuh"

namespace pipo {

namespace {

template <int DH, bool PAIR, bool SEL>
cudaError_t tile_as(const AttnPagedArgs& a, const AttnPlan& pl, const CUtensorMap& tk, const CUtensorMap& tv,
                    cudaStream_t s) {
    auto* fn = &attn_tile_kernel<DH, PAIR, SEL>;
    static thread_local int ready_dev = -1;  // the shared-memory limit is set per device
    if (ready_dev != pl.dev) {
        const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)at_smem(DH, PAIR));
        if (e != cudaSuccess) return e;
        ready_dev = pl.dev;
    }
    const ItemShape shape{pl.TP, a.window, pl.listed ? a.n_top : 0};
    const cudaError_t e = launch_pdl(fn, dim3((unsigned)pl.ctas), kAtThreads, at_smem(DH, PAIR), s, a, shape, pl.workers,
                                     pl.part_rows, pl.part_off, tk, tv);
    return e == cudaSuccess ? launch_combine<DH, bf16_t>(a, pl, s) : e;
}

}  // namespace

// The plan of a launch; scratch: see work.cuh.
// bf16: pairs of row tiles when the sequences of the batch have more than 128 rows
// on average.  fp32: tiles of 64 rows when they have more than 16, else of 16.
// n_top > 0: attention over selected pages (< 0: by lists, whatever the sizes).  By lists a token and
// kv head read n_top pages; a tile of tokens reads every page up to its last position once
// for all of them and masks by bits.  Whole tiles, when the tokens of a sequence (on average, a
// tile's at most) times n_top reach max_pages: such a tile reads no more than its tokens' lists
// name.  (bf16, 512 tokens with 16 of 249 pages each: 279 us by lists, 143 by tiles at that time.)
// The lengths are on the device, so the rule goes by the batch's average and the table's width:
// decoding sequences beside a long chunk read all their pages with it, and a chunk under a table much
// wider than its cache, or beside many idle sequences, goes by lists.  Either way the same
// pages have weight.
AttnPlan plan_attn(const PagedArgs& c, int n_top, int dev, int sms) {
    AttnPlan pl{};
    pl.dev = dev;
    const long long mine = (long long)c.n_tokens * c.G;
    const bool chunks = mine > 128LL * c.batch;
    if (n_top < 0) pl.listed = true;
    if (n_top > 0) {
        const long long tokens = c.n_tokens / c.batch, tile = 256 / c.G;
        pl.listed = !(c.dtype && chunks && (tokens < tile ? tokens : tile) * n_top >= c.max_pages);
    }
    const bool listed = pl.listed;
    int rows, per;  // rows of a tile, workers of an SM
    if (c.dtype) {
        pl.pair = !listed && chunks;
        rows = pl.pair ? 256 : 128;
        per = pl.pair ? 1 : 2;
    } else {
        pl.rt = !listed && mine > 16LL * c.batch ? 4 : 1;
        rows = af_rows(pl.rt);
        per = af_ctas(c.dh, pl.rt);
    }
    pl.TP = listed ? 1 : rows / c.G;
    pl.tiles = tiles_bound(c.n_tokens, c.batch, pl.TP);
    const long long each = (c.max_pages + 1) / 2, most = pl.tiles * c.n_kv * each;  // units of an item, in all, at most
    pl.workers = (int)(most < (long long)sms * per ? most : (long long)sms * per);
    const int cta_workers = c.dtype && !pl.pair ? 2 : 1;
    pl.ctas = (pl.workers + cta_workers - 1) / cta_workers;
    pl.workers = pl.ctas * cta_workers;
    pl.join = each > 1;  // items of one unit are nobody's in part
    pl.part_rows = (int)(mine < (long long)pl.TP * c.G ? mine : (long long)pl.TP * c.G);
    pl.part_rows += pl.part_rows & 1;
    pl.part_off = record_bytes(pl.workers);
    pl.bits_off = pl.part_off + (size_t)pl.workers * 2 * part_floats(pl.part_rows, c.dh) * sizeof(float);
    pl.scratch = pl.bits_off;
    if (n_top > 0 && !listed) pl.scratch += (size_t)c.n_tokens * c.n_kv * bit_words(c.max_pages) * 4;
    return pl;
}

cudaError_t launch_attn_tile(const AttnPagedArgs& a, const AttnPlan& pl, const CUtensorMap& tk, const CUtensorMap& tv,
                             cudaStream_t s) {
    if (a.c.dh == 64)
        return !pl.pair ? tile_as<64, false, false>(a, pl, tk, tv, s)
               : a.bits ? tile_as<64, true, true>(a, pl, tk, tv, s)
                        : tile_as<64, true, false>(a, pl, tk, tv, s);
    return !pl.pair ? tile_as<128, false, false>(a, pl, tk, tv, s)
           : a.bits ? tile_as<128, true, true>(a, pl, tk, tv, s)
                    : tile_as<128, true, false>(a, pl, tk, tv, s);
}

cudaError_t take_error_paged(unsigned* code, unsigned* info) { return take_unit_error(code, info); }

}  // namespace pipo
