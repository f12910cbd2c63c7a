// Attention over lists of pages: a list for `run` new tokens of a sequence and a KV head.
// The rows of a run and its list take the place of a sequence's rows and keys in the
// kernels of the whole cache; a page of the list is anywhere in the sequence, so its first
// key is read beside its number.
//
// Measured at d = 128, 32/8 heads: single tokens of 16 sequences on lists of 32 pages of 128 keys 31.7 us
// (28.5 for 134 MB of K and V, 4.7 TB/s, and 4 for the merge); of one sequence on 128 pages of 64, E4M3
// queries, 13.9; 2048 tokens in runs of 32 on 32 pages each 114 to 124 us, 1.11 to 1.20 PFLOP/s.
#include "cache_merge.hpp"

namespace attn {

FwdPlan blocks_plan(int64_t lists, int G, int run, int take, int page, int d, int n_cu)
{
    const int visits = (take + kVisit / page - 1) / (kVisit / page);
    FwdPlan pl = cache_fwd_plan(lists, (int64_t)run * G, visits, d, n_cu, true);
    // few lists: a visit for each wave, where that leaves CUs free all the same (8 lists x 64 visits
    // 18.0 -> 14.7 us, 26 x 33 18.8 -> 17.3, 28 x 26 at d = 64 14.1 -> 13.9; not so 32 x 32, 17.3 -> 18.9)
    const int64_t units = lists * pl.tiles, ranges = (visits + 3) / 4;
    if (pl.rows == 16 && pl.ranges > 1 && pl.chunk == 8 && units * ranges < n_cu) {
        pl.chunk = 4;
        pl.ranges = (int)ranges;
        pl.bytes = (size_t)units * ranges * pl.rows * (d + 2) * sizeof(float);
    } else if (pl.ranges == 2 && (pl.rows == 16 ? visits <= (d == 64 ? 24 : 16) : visits <= 16 && (int64_t)run * G > 64)) {
        // short lists: no merge (16-row tiles: 160 lists x 10 visits at d = 64 17.1 -> 13.7 us, 208 x 21 21.5 -> 18.6; at
        // d = 128 96 x 9 17.4 -> 16.2, 112 x 16 18.9 -> 18.2; 128-row tiles: 256 lists x 128 rows x 5 38.6 -> 23.1, 224 x 128 x 14
        // 49.3 -> 45.9; not so 216 x 64 x 8, 32.3 -> 32.5)
        pl.chunk = visits;
        pl.ranges = 1;
        pl.bytes = 0;
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
