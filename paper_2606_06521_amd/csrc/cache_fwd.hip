// Attention of new tokens over the cache: plan, launch, merge.
#include "cache_fwd_tile.hpp"

#include <algorithm>
#include <cmath>

namespace attn {

namespace {

// Ranges of a tile at most: 2^26 keys in ranges of kMaxChunk visits.
constexpr int kMergeRanges = 4096;
static_assert((1 << 26) / kVisit / kMaxChunk <= kMergeRanges && kTileChunk >= kMaxChunk);

// Merge of a split tile: PARTS * D / 4 threads per query row, thread (piece, part)
// takes one 16-byte piece of the row from every PARTS-th range; the parts are
// added through LDS in a fixed order.  Ranges stand at their own power of two; the
// row's is the largest.  Many ranges: a row per workgroup (latency: all references
// at once, then all partial sums); few: a row per D / 4 threads.
template <int D, int PARTS>
__global__ void __launch_bounds__(256) cache_merge(FwdParams p, int tile_rows)
{
    constexpr int PIECES = D / 4, RPW = 256 / (PIECES * PARTS);
    static_assert(RPW == 1 || PARTS == 1, "a workgroup's rows end at different places");
    __shared__ f32x4 osh[RPW][PARTS][PIECES];
    __shared__ float lsh[RPW][PARTS], msh[PARTS > 1 ? kMergeRanges : 1], wave_max[4];
    const int per_seq = p.bt.max_q * p.gr.G, groups = (per_seq + RPW - 1) / RPW;
    const int64_t unit = blockIdx.x / groups;
    const int hk = (int)(unit % p.cache.Hkv), b = (int)(unit / p.cache.Hkv);
    const int sub = threadIdx.x / (PIECES * PARTS);
    const int R = (int)(blockIdx.x - unit * groups) * RPW + sub;
    const Seq s = sequence(p.bt, b, p.max_len);
    if (R >= s.n * p.gr.G)
        return;
    const int tile = R / tile_rows;
    const int n = (tile_visits(p, s, tile, tile_rows) + p.chunk - 1) / p.chunk;
    if (n <= 1)
        return;                                  // (the range wrote the row itself)
    const int rr = R - tile * tile_rows;
    const size_t stride = (size_t)tile_rows * (D + 2);
    const float* base = p.ws + (((size_t)b * p.cache.Hkv + hk) * p.tiles + tile) * p.ranges * stride;
    const int piece = threadIdx.x % PIECES, part = threadIdx.x / PIECES % PARTS;
    float m = -INFINITY;
    if constexpr (PARTS > 1) {
        for (int c = threadIdx.x; c < n; c += 256) {
            const float x = base[c * stride + tile_rows * (D + 1) + rr];
            msh[c] = x;
            m = fmax_f(m, x);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1)
            m = fmax_f(m, __shfl_xor(m, off, 64));
        m = halves_max(m);
        if ((threadIdx.x & 63) == 0)
            wave_max[threadIdx.x >> 6] = m;
        __syncthreads();
        m = fmax_f(fmax_f(wave_max[0], wave_max[1]), fmax_f(wave_max[2], wave_max[3]));
    } else {
#pragma unroll 4
        for (int c = 0; c < n; ++c)
            m = fmax_f(m, base[c * stride + tile_rows * (D + 1) + rr]);
    }
    f32x4 acc = {};
    float l = 0.f;
#pragma unroll 4
    for (int c = part; c < n; c += PARTS) {
        const float* at = base + c * stride;
        const f32x4 x = *reinterpret_cast<const f32x4*>(at + rr * D + 4 * piece);
        const float lc = at[tile_rows * D + rr], mc = PARTS > 1 ? msh[c] : at[tile_rows * (D + 1) + rr];
        const int down = shift_of(mc, m);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc[e] += __builtin_amdgcn_ldexpf(x[e], down);
        l += __builtin_amdgcn_ldexpf(lc, down);
    }
    if constexpr (PARTS > 1) {
        osh[sub][part][piece] = acc;
        if (piece == 0)
            lsh[sub][part] = l;
        __syncthreads();
        if (part != 0)
            return;
#pragma unroll
        for (int v = 1; v < PARTS; ++v) {
            const f32x4 t = osh[sub][v][piece];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[e] += t[e];
            l += lsh[sub][v];
        }
    }
    write_row<D>(p, s, hk, R, piece, acc, l, 1.f / l, m);
}

template <int D, int PAGE>
hipError_t fwd_go(const FwdParams& p, int rows, bool e4m3, unsigned grid, hipStream_t s)
{
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    if (rows == kTileRows)
        return e4m3 ? go(cache_fwd_tile_kernel<D, PAGE, true>) : go(cache_fwd_tile_kernel<D, PAGE, false>);
    return e4m3 ? go(cache_fwd_kernel<D, PAGE, true>) : go(cache_fwd_kernel<D, PAGE, false>);
}

// Time of a call on tiles of 16 or of 128 rows, in units of a microsecond, and its plan.
//   16 rows:  a workgroup per CU (two at d = 64), whose four waves take a visit each; a
//             wave's visit takes 3 of them at d = 128
//   128 rows: two workgroups per CU, each of them a visit at a time: 4.1 in company, 2.5 alone
// (at d = 64 0.6 of both), a workgroup's first loads and last sum 6 or 9, and where a tile is split its
// merge: a launch, and the partial sums written and read.  Measured at 16 x 8 heads x
// 8192 keys: 32 rows 51 (16-row tiles) against 82, 96 rows 149 against 113; one
// sequence x 8 heads x 32768 keys: 64 rows 33 against 46, 256 rows 94 against 61.
double plan_time(FwdPlan& pl, int rows, int64_t heads, int64_t run, int visits, int d, int n_cu)
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
    const double visit = (d == 64 ? 0.6 : 1.0) * (tall ? (wgs > n_cu ? 4.1 : 2.5) : 3.0 * (slots > n_cu && wgs > n_cu ? 1.5 : 1.0) / 4);
    return 2 + rounds * ((tall ? 9 : 6) + each * visit) + (pl.ranges > 1 ? 5 + 2e-6 * pl.bytes / 2.5 : 0);
}

}  // namespace

FwdPlan cache_fwd_plan(int B, int Hkv, int G, int max_q, int max_len, int d, int n_cu)
{
    FwdPlan low, tall;
    const int64_t heads = (int64_t)B * Hkv, run = (int64_t)max_q * G;
    const int visits = (max_len + kVisit - 1) / kVisit;
    const double t_low = plan_time(low, 16, heads, run, visits, d, n_cu);
    return run > 16 && plan_time(tall, kTileRows, heads, run, visits, d, n_cu) < t_low ? tall : low;
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
    e = d == 64 ? (page == 64 ? fwd_go<64, 64>(p, pl.rows, e4m3, g.tiles, s) : fwd_go<64, 128>(p, pl.rows, e4m3, g.tiles, s))
                : (page == 64 ? fwd_go<128, 64>(p, pl.rows, e4m3, g.tiles, s) : fwd_go<128, 128>(p, pl.rows, e4m3, g.tiles, s));
    if (e == hipSuccess && pl.ranges > 1) {
        auto merge = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(g.merges), dim3(256), 0, s, p, pl.rows); };
        if (d == 64)
            g.merge_rows == 1 ? merge(cache_merge<64, 16>) : merge(cache_merge<64, 1>);
        else
            g.merge_rows == 1 ? merge(cache_merge<128, 8>) : merge(cache_merge<128, 1>);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace attn
