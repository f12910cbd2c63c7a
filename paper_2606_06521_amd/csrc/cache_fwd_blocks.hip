// Attention over lists of pages: a list for `run` new tokens of a sequence and a KV head.
// The rows of a run and its list take the place of a sequence's rows and keys in the
// kernels of the whole cache; a page of the list is anywhere in the sequence, so its first
// key is read beside its number.
//
// Measured at d = 128, 32/8 heads: single tokens of 16 sequences on lists of 32 pages of 128 keys 32.9 us
// (28.5 for 134 MB of K and V, 4.7 TB/s, and 4.5 for the merge); of one sequence on 128 pages of 64, E4M3
// queries, 13.8; 2048 tokens in runs of 32 on 32 pages each 117 us, 1.17 PFLOP/s.
#include "cache_merge.hpp"

namespace attn {

FwdPlan blocks_plan(int64_t lists, int G, int run, int take, int page, int d, int n_cu)
{
    const int visits = (take + kVisit / page - 1) / (kVisit / page);
    FwdPlan pl = cache_fwd_plan(lists, (int64_t)run * G, visits, d, n_cu);
    // few lists: a visit for each wave, where that leaves every second CU free all the same (8 lists x 64 visits
    // 18.0 -> 14.7 us, 8 x 32 14.6 -> 13.6; not so 32 x 32, 17.3 -> 18.9)
    const int64_t units = lists * pl.tiles, ranges = (visits + 3) / 4;
    if (pl.rows == 16 && pl.ranges > 1 && pl.chunk == 8 && units * ranges <= n_cu / 2) {
        pl.chunk = 4;
        pl.ranges = (int)ranges;
        pl.bytes = (size_t)units * ranges * pl.rows * (d + 2) * sizeof(float);
    }
    return pl;
}

hipError_t blocks_grids(int64_t lists, int64_t rows, int d, const FwdPlan& pl, FwdGrids& g)
{
    const hipError_t e = grid_of(((__int128)lists * pl.tiles * pl.ranges + kNumXcd - 1) / kNumXcd * kNumXcd, 256, g.tiles);
    g.merge_rows = pl.ranges > 8 ? 1 : 1024 / d;
    g.merges = 0;
    return e != hipSuccess || pl.ranges == 1 ? e : grid_of((__int128)lists * ((rows + g.merge_rows - 1) / g.merge_rows), 256, g.merges);
}

hipError_t launch_cache_fwd_blocks(BlocksParams p, const FwdPlan& pl, int d, int page, bool e4m3, hipStream_t s)
{
    p.tiles = pl.tiles;
    p.chunk = pl.chunk;
    p.ranges = pl.ranges;
    FwdGrids g;
    hipError_t e = blocks_grids((int64_t)p.bt.B * p.cache.Hkv * p.runs, (int64_t)p.run * p.gr.G, d, pl, g);
    if (e != hipSuccess)
        return e;
    e = fwd_launch(p, pl.rows, d, page, e4m3, g.tiles, s);
    return e == hipSuccess && pl.ranges > 1 ? merge_launch(p, pl.rows, d, page, g.merges, g.merge_rows, s) : e;
}

}  // namespace attn
