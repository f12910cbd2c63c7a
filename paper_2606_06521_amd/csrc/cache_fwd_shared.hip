// Attention of a batch whose sequences begin with the same pages.
//
// A group of keys has its own power of two, so the partial sums of any parts of the keys
// add up to the whole cache's result.  The shared pages are one part: the queries of all
// sequences are the rows of its tiles, so that each of its keys is read once and meets
// B G n rows instead of G n.  What follows in each sequence is the other part.
//
// Measured at d = 128, 32/8 heads: single tokens of 32 sequences behind 16384 common keys and up to 1024 of their own
// 28.7 us (72 MB read; 23 for both kinds of tile in one launch, 6 for the merge); chunks of up to 192
// tokens of 8 such sequences 206 to 214 us, 1.06 to 1.11 PFLOP/s (196 in the tiles, 13 for the merge, which
// reads 44 MB).
#include "cache_merge.hpp"

#include <algorithm>
#include <cmath>

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

// Plan of the shared pages where the sequences' own take 16-row tiles, by modelled time in microseconds:
//   16-row tiles, a workgroup per CU (two at d = 64): 11.5 (9.2 at d = 64), 0.48 for each visit of a workgroup (0.62 where
//     they fill the GPU) and 0.15 for each range that a row's merge adds up; for each further round of
//     workgroups 6 and 0.75 for each visit of the own pages;
//   128-row tiles in the same launch: 10, 0.29 for each MB of partial results, and of the two that run at once, a workgroup's
//     own visits, 2.1 each, and what all of them take of the GPU (0.006 for each visit, 0.0056 for each workgroup,
//     for each of the own pages' 0.007 and 0.0033 for each of its visits), the root of the sum of their cubes
// (0.7 of a visit at d = 64, 0.74 on 128-row tiles).  Over 600 calls (2 to 256 sequences, 256 to 92000 shared keys, 16 to
// 6000 own ones, 1 to 64 tokens, 1 to 16 KV heads of 1 to 8 rows) the plan takes 1.05 times the best
// one's time, 1.14 in nine of ten, 1.49 at most.  Measured with 300 own tokens and 32/8 heads at d = 128: 4 sequences x 16384
// shared keys 18.9 (16-row tiles) against 20.4, 16 x 16384 27.3 against 23.1, 64 x 16384 58 against 37;
// 32 x 2048 19.6 against 18.8; 16 x 16/2 heads x 8192 15.4 against 17.5.
FwdPlan shared_pages_plan(int Hkv, int64_t rows, int visits, int64_t own_wgs, int own_visits, int d, int n_cu)
{
    const double f = d == 64 ? 0.7 : 1.0;
    FwdPlan best{};
    double t_best = 0;
    for (const int tile : {16, kTileRows}) {
        const bool tall = tile == kTileRows;
        const int64_t tiles = (rows + tile - 1) / tile;
        for (int chunk = tall ? 2 : 8;; chunk *= 2) {
            chunk = std::min(chunk, tall ? kTileChunk : kMaxChunk);
            const int ranges = std::max(1, (visits + chunk - 1) / chunk);
            const double wgs = (double)Hkv * tiles * ranges, each = std::min(chunk, visits);
            const double mb = 1e-6 * wgs * tile * (d + 2) * sizeof(float);
            const double slots = n_cu * (d == 64 ? 2.0 : 1.0);
            double t;
            if (tall) {
                const double f8 = d == 64 ? 0.74 : 1.0, own = 2.1 * f8 * each;
                const double all = 256.0 / n_cu * (0.006 * f8 * Hkv * tiles * visits + 0.0056 * wgs + own_wgs * (0.007 + 0.0033 * f8 * own_visits));
                t = 10 + 0.29 * mb + std::cbrt(own * own * own + all * all * all);
            } else {
                t = (d == 64 ? 9.2 : 11.5) + f * each * (wgs < 0.75 * slots ? 0.48 : 0.62 * std::max(1.0, std::floor(wgs / slots))) +
                    0.15 * ranges + (6 + 0.75 * f * own_visits) * (std::ceil((wgs + own_wgs) / slots) - 1);
            }
            if (!best.rows || t < t_best) {
                t_best = t;
                best = {tile, (int)tiles, chunk, ranges, 0};
            }
            if (chunk >= visits || chunk == (tall ? kTileChunk : kMaxChunk))
                break;
        }
    }
    return best;
}

}  // namespace

SharedPlan shared_plan(int B, int Hkv, int G, int T, int max_q, int shared, int max_len, int page, int d, int n_cu)
{
    const int base = (int)std::min<int64_t>((int64_t)shared * page, max_len), visits = (base + kVisit - 1) / kVisit;
    const int own_visits = (max_len - base + kVisit - 1) / kVisit;
    const int64_t rows = (int64_t)T * G;
    SharedPlan pl;
    pl.own = cache_fwd_plan((int64_t)B * Hkv, (int64_t)max_q * G, own_visits, d, n_cu);
    pl.pre = pl.own.rows == kTileRows
                 ? cache_fwd_plan(Hkv, rows, visits, d, n_cu)
                 : shared_pages_plan(Hkv, rows, visits, (int64_t)B * Hkv * pl.own.tiles * pl.own.ranges, std::min(pl.own.chunk, own_visits), d, n_cu);
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
