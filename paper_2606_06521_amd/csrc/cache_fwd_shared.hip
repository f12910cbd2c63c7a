// Attention of a batch whose sequences begin with the same pages.
//
// A group of keys has its own power of two, so the partial sums of any parts of the keys
// add up to the whole cache's result.  The shared pages are one part: the queries of all
// sequences are the rows of its tiles, so that each of its keys is read once and meets
// B G n rows instead of G n.  What follows in each sequence is the other part.
#include "cache_merge.hpp"

#include <algorithm>

namespace attn {

namespace {

hipError_t both_launch(const SharedParams& p, int d, int page, bool e4m3, unsigned grid, hipStream_t s)
{
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    if (d == 64)
        return page == 64 ? (e4m3 ? go(cache_fwd_both_kernel<64, 64, true>) : go(cache_fwd_both_kernel<64, 64, false>))
                          : (e4m3 ? go(cache_fwd_both_kernel<64, 128, true>) : go(cache_fwd_both_kernel<64, 128, false>));
    return page == 64 ? (e4m3 ? go(cache_fwd_both_kernel<128, 64, true>) : go(cache_fwd_both_kernel<128, 64, false>))
                      : (e4m3 ? go(cache_fwd_both_kernel<128, 128, true>) : go(cache_fwd_both_kernel<128, 128, false>));
}

}  // namespace

SharedPlan shared_plan(int B, int Hkv, int G, int T, int max_q, int shared, int max_len, int page, int d, int n_cu)
{
    const int base = (int)std::min<int64_t>((int64_t)shared * page, max_len);
    SharedPlan pl;
    pl.pre = cache_fwd_plan(Hkv, (int64_t)T * G, (base + kVisit - 1) / kVisit, d, n_cu);
    pl.own = cache_fwd_plan((int64_t)B * Hkv, (int64_t)max_q * G, (max_len - base + kVisit - 1) / kVisit, d, n_cu);
    pl.pre.bytes = (size_t)Hkv * pl.pre.tiles * pl.pre.ranges * pl.pre.rows * (d + 2) * sizeof(float);
    pl.own.bytes = (size_t)B * Hkv * pl.own.tiles * pl.own.ranges * pl.own.rows * (d + 2) * sizeof(float);
    return pl;
}

hipError_t shared_grids(int B, int Hkv, int G, int max_q, int d, const SharedPlan& pl, SharedGrids& g)
{
    auto whole = [](__int128 wgs) { return (wgs + kNumXcd - 1) / kNumXcd * kNumXcd; };
    const __int128 pre = whole((__int128)Hkv * pl.pre.tiles * pl.pre.ranges);
    const __int128 own = whole((__int128)B * Hkv * pl.own.tiles * pl.own.ranges);
    unsigned both;
    hipError_t e = pl.pre.ranges + pl.own.ranges <= kSharedRanges ? grid_of(pre, 256, g.pre) : hipErrorNotSupported;
    if (e == hipSuccess)
        e = grid_of(own, 256, g.own);
    if (e == hipSuccess)
        e = grid_of(pre + own, 256, both);
    g.merge_rows = pl.pre.ranges + pl.own.ranges > 8 ? 1 : 1024 / d;
    return e != hipSuccess ? e : grid_of((__int128)B * Hkv * (((int64_t)max_q * G + g.merge_rows - 1) / g.merge_rows), 256, g.merges);
}

hipError_t launch_cache_fwd_shared(SharedParams p, const SharedPlan& pl, int d, int page, bool e4m3, hipStream_t s)
{
    p.tiles = pl.own.tiles;
    p.chunk = pl.own.chunk;
    p.ranges = pl.own.ranges;
    p.pre_tiles = pl.pre.tiles;
    p.pre_chunk = pl.pre.chunk;
    p.pre_ranges = pl.pre.ranges;
    p.pre_rows = pl.pre.rows;
    p.pre_ws = p.ws;
    p.ws += pl.pre.bytes / sizeof(float);
    SharedGrids g;
    hipError_t e = shared_grids(p.bt.B, p.cache.Hkv, p.gr.G, p.bt.max_q, d, pl, g);
    if (e != hipSuccess)
        return e;
    p.pre_grid = g.pre;
    if (pl.pre.rows == pl.own.rows) {
        e = fwd_launch(p, pl.pre.rows, d, page, e4m3, g.pre + g.own, s);
    } else if (pl.pre.rows == kTileRows) {
        e = both_launch(p, d, page, e4m3, g.pre + g.own, s);
    } else {
        e = fwd_launch(p, pl.pre.rows, d, page, e4m3, g.pre, s);
        p.pre_grid = 0;
        if (e == hipSuccess)
            e = fwd_launch(p, pl.own.rows, d, page, e4m3, g.own, s);
    }
    return e == hipSuccess ? merge_launch(p, pl.own.rows, d, page, g.merges, g.merge_rows, s) : e;
}

}  // namespace attn
