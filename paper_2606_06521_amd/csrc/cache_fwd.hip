// Attention of new tokens over the cache: plan, launch, merge.
#include "cache_merge.hpp"

#include <algorithm>
#include <cmath>

namespace attn {

namespace {

// Time of a call on tiles of 16 or of 128 rows, in units of a microsecond, and its plan.
//   16 rows:  a workgroup per CU (two at d = 64), whose four waves take a visit each; a
//             wave's visit takes 3 of them at d = 128
//   128 rows: two workgroups per CU, each of them a visit at a time: 4.1 in company, 2.5 alone
// (at d = 64 0.6 of both), a workgroup's first loads and last sum 6 or 9, and where a tile is split its
// merge: a launch, and the partial sums written and read.  Measured at 16 x 8 heads x
// 8192 keys: 32 rows 51 (16-row tiles) against 82, 96 rows 149 against 113; one
// sequence x 8 heads x 32768 keys: 64 rows 33 against 46, 256 rows 94 against 61.
// Lists of neighbouring runs share pages, so their 128-row tiles wait less for memory: a visit takes 2.3 (at
// d = 64 0.6 of 2.8) where one wave has rows, 3.0 where two have, and partial sums are read back from the caches.
// d = 128: 2560 lists x 32 rows x 15 visits 213 against 328 on 16-row tiles, 512 x 32 x 121 301 against 293;
// d = 64: 448 x 32 x 43 82 against 56.
double plan_time(FwdPlan& pl, int rows, int64_t heads, int64_t run, int visits, int d, int n_cu, bool lists)
{
    const bool tall = rows == kTileRows;
    pl.rows = rows;
    pl.tiles = (int)((run + rows - 1) / rows);
    const int64_t units = heads * pl.tiles, slots = (int64_t)n_cu * (tall || d == 64 ? 2 : 1);
    // enough ranges to fill the GPU, none shorter than two visits of each wave, or
    // four of a tall tile's
    const int64_t want = std::min<int64_t>(std::max<int64_t>(1, slots / std::max<int64_t>(units, 1)), kMergeRanges);
    pl.chunk = (int)std::max<int64_t>(tall ? 4 : 8, (visits + want - 1) / want);
    pl.chunk = std::min(pl.chunk, tall ? kTileChunk : kMaxChunk);
    pl.ranges = std::max(1, (visits + pl.chunk - 1) / pl.chunk);
    pl.bytes = pl.ranges > 1 ? (size_t)units * pl.ranges * rows * (d + 2) * sizeof(float) : 0;
    const double wgs = (double)units * pl.ranges, rounds = std::ceil(wgs / slots), each = std::min(pl.chunk, visits);
    const double beside = !lists || run > 64 ? 4.1 : run > 32 ? 3.0 : d == 64 ? 2.8 : 2.3;
    const double visit = (d == 64 ? 0.6 : 1.0) * (tall ? (wgs > n_cu ? beside : std::min(beside, 2.5)) : 3.0 * (slots > n_cu && wgs > n_cu ? 1.5 : 1.0) / 4);
    return 2 + rounds * ((tall ? 9 : 6) + each * visit) + (pl.ranges > 1 ? 5 + (lists ? 0.29e-6 : 0.8e-6) * pl.bytes : 0);
}

}  // namespace

FwdPlan cache_fwd_plan(int64_t heads, int64_t rows, int visits, int d, int n_cu, bool lists)
{
    FwdPlan low, tall;
    const double t_low = plan_time(low, 16, heads, rows, visits, d, n_cu, lists);
    return rows > 16 && plan_time(tall, kTileRows, heads, rows, visits, d, n_cu, lists) < t_low ? tall : low;
}

FwdPlan cache_fwd_plan(int B, int Hkv, int G, int max_q, int max_len, int d, int n_cu)
{
    return cache_fwd_plan((int64_t)B * Hkv, (int64_t)max_q * G, (max_len + kVisit - 1) / kVisit, d, n_cu);
}

bool cache_fwd_fits(int B, int Hkv, int G, int max_q)
{
    unsigned grid;
    return grid_of((__int128)B * Hkv * (((int64_t)max_q * G + kTileRows - 1) / kTileRows), 256, grid) == hipSuccess;
}

hipError_t cache_fwd_grids(int B, int Hkv, int G, int max_q, int d, const FwdPlan& pl, FwdGrids& g)
{
    const int64_t heads = (int64_t)B * Hkv;
    // whole rounds of the XCDs
    const hipError_t e = grid_of(((__int128)heads * pl.tiles * pl.ranges + kNumXcd - 1) / kNumXcd * kNumXcd, 256, g.tiles);
    // rows of a merging workgroup: one, or as many as have a thread per 16 bytes
    g.merge_rows = pl.ranges > 8 ? 1 : 1024 / d;
    g.merges = 0;
    return e != hipSuccess || pl.ranges == 1
               ? e
               : grid_of((__int128)heads * (((int64_t)max_q * G + g.merge_rows - 1) / g.merge_rows), 256, g.merges);
}

hipError_t launch_cache_fwd(FwdParams p, const FwdPlan& pl, int d, int page, bool e4m3, hipStream_t s)
{
    p.tiles = pl.tiles;
    p.chunk = pl.chunk;
    p.ranges = pl.ranges;
    FwdGrids g;
    hipError_t e = cache_fwd_grids(p.bt.B, p.cache.Hkv, p.gr.G, p.bt.max_q, d, pl, g);
    if (e != hipSuccess)
        return e;
    e = fwd_launch(p, pl.rows, d, page, e4m3, g.tiles, s);
    return e == hipSuccess && pl.ranges > 1 ? merge_launch(p, pl.rows, d, page, g.merges, g.merge_rows, s) : e;
}

}  // namespace attn
