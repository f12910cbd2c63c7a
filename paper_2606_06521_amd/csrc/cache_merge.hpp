// The attention's launches by head size, page and type, and the merge of split tiles.
#pragma once

#include "cache_fwd_tile.hpp"

namespace attn {

namespace {

// Ranges of a tile at most: 2^26 keys in ranges of kMaxChunk visits.
constexpr int kMergeRanges = 4096;
// Of a row of the shared call, both kinds: as many, and what is split to fill the GPU.
constexpr int kSharedRanges = kMergeRanges + 1024;
static_assert((1 << 26) / kVisit / kMaxChunk <= kMergeRanges && kTileChunk >= kMaxChunk);

// Query rows of a unit.
__device__ inline int rows_of(const FwdParams& p) { return p.bt.max_q * p.gr.G; }
__device__ inline int rows_of(const BlocksParams& p) { return p.run * p.gr.G; }

// The partial results of a query row: those of the shared pages' ranges, if there are, then
// those of its own tile's.
struct RowParts {
    struct One {
        const float *o, *l, *m;
    };
    struct Run {
        const float* base;
        int n, rows, row, d;
        __device__ inline One at(int c) const
        {
            const float* const x = base + (size_t)c * rows * (d + 2);
            return {x + row * d, x + rows * d + row, x + rows * (d + 1) + row};
        }
    };
    Run pre, own;
    int n;
    __device__ inline One at(int c) const { return c < pre.n ? pre.at(c) : own.at(c - pre.n); }
};

template <class P>
__device__ inline RowParts parts_of(const P& p, const Unit& u, int unit, int R, int tile_rows, int page, int d)
{
    RowParts a{};
    const int tile = R / tile_rows;
    a.own = {p.ws + ((size_t)unit * p.tiles + tile) * p.ranges * ((size_t)tile_rows * (d + 2)), p.ranges, tile_rows,
             R - tile * tile_rows, d};
    if constexpr (!kLists<P>)
        a.own.n = (tile_visits(p, u, tile, tile_rows, page) + p.chunk - 1) / p.chunk;
    if constexpr (kShared<P>) {
        const Unit all = unit_of(p, u.hk, true);
        const int row = u.s.first * p.gr.G + R, at = row / p.pre_rows;
        a.pre = {p.pre_ws + ((size_t)u.hk * p.pre_tiles + at) * p.pre_ranges * ((size_t)p.pre_rows * (d + 2)),
                 (tile_visits(p, all, at, p.pre_rows, page) + p.pre_chunk - 1) / p.pre_chunk, p.pre_rows, row - at * p.pre_rows, d};
    }
    a.n = a.pre.n + a.own.n;
    return a;
}

// Merge of a split tile: PARTS * D / 4 threads per query row, thread (piece, part)
// takes one 16-byte piece of the row from every PARTS-th range; the parts are
// added through LDS in a fixed order.  Ranges stand at their own power of two; the
// row's is the largest.  Many ranges: a row per workgroup (latency: all references
// at once, then all partial sums); few: a row per D / 4 threads.
template <int D, int PARTS, class P>
__global__ void __launch_bounds__(256) cache_merge(P p, int tile_rows, int page)
{
    constexpr int PIECES = D / 4, RPW = 256 / (PIECES * PARTS);
    static_assert(RPW == 1 || PARTS == 1, "a workgroup's rows end at different places");
    constexpr int MOST = kShared<P> ? kSharedRanges : kMergeRanges;
    __shared__ f32x4 osh[RPW][PARTS][PIECES];
    __shared__ float lsh[RPW][PARTS], msh[PARTS > 1 ? MOST : 1], wave_max[4];
    const int per_unit = rows_of(p), groups = (per_unit + RPW - 1) / RPW;
    const int unit = (int)(blockIdx.x / groups);
    const int sub = threadIdx.x / (PIECES * PARTS);
    const int R = (int)(blockIdx.x - (unsigned)unit * groups) * RPW + sub;
    const Unit u = unit_of(p, unit, false);
    const Seq& s = u.s;
    if (R >= s.n * p.gr.G)
        return;
    const RowParts a = parts_of(p, u, unit, R, tile_rows, page, D);
    const int n = a.n;
    if (!kShared<P> && n <= 1)
        return;                                  // (the range wrote the row itself)
    const int piece = threadIdx.x % PIECES, part = threadIdx.x / PIECES % PARTS;
    float m = -INFINITY;
    // few parts: all of them on their way at once (references first and then the sums: 4.0 us in the place of 3.2 for 32
    // rows of two parts, 15.9 in the place of 13.8 for 27200 of three)
    constexpr int FEW = 4;
    if (PARTS == 1 && n <= FEW) {
        f32x4 x[FEW], acc = {};
        float lc[FEW], mc[FEW], l = 0.f;
#pragma unroll
        for (int c = 0; c < FEW; ++c) {
            const RowParts::One r = a.at(max(min(c, n - 1), 0));
            x[c] = *reinterpret_cast<const f32x4*>(r.o + 4 * piece);
            lc[c] = *r.l;
            mc[c] = *r.m;
        }
#pragma unroll
        for (int c = 0; c < FEW; ++c)
            m = c < n ? fmax_f(m, mc[c]) : m;
#pragma unroll
        for (int c = 0; c < FEW; ++c) {
            if (c >= n)
                continue;
            const int down = shift_of(mc[c], m);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[e] += __builtin_amdgcn_ldexpf(x[c][e], down);
            l += __builtin_amdgcn_ldexpf(lc[c], down);
        }
        write_row<D>(p, s, u.hk, R, piece, acc, l, 1.f / l, m);
        return;
    }
    if constexpr (PARTS > 1) {
        for (int c = threadIdx.x; c < n; c += 256) {
            const float x = *a.at(c).m;
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
            m = fmax_f(m, *a.at(c).m);
    }
    f32x4 acc = {};
    float l = 0.f;
#pragma unroll 4
    for (int c = part; c < n; c += PARTS) {
        const RowParts::One r = a.at(c);
        const f32x4 x = *reinterpret_cast<const f32x4*>(r.o + 4 * piece);
        const float lc = *r.l, mc = PARTS > 1 ? msh[c] : *r.m;
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
    write_row<D>(p, s, u.hk, R, piece, acc, l, 1.f / l, m);
}

template <class P, int D, int PAGE>
hipError_t fwd_launch_of(const P& p, int rows, bool e4m3, unsigned grid, hipStream_t s)
{
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    if (rows == kTileRows)
        return e4m3 ? go(cache_fwd_tile_kernel<D, PAGE, true, P>) : go(cache_fwd_tile_kernel<D, PAGE, false, P>);
    return e4m3 ? go(cache_fwd_kernel<D, PAGE, true, P>) : go(cache_fwd_kernel<D, PAGE, false, P>);
}

template <class P>
hipError_t fwd_launch(const P& p, int rows, int d, int page, bool e4m3, unsigned grid, hipStream_t s)
{
    return d == 64 ? (page == 64 ? fwd_launch_of<P, 64, 64>(p, rows, e4m3, grid, s) : fwd_launch_of<P, 64, 128>(p, rows, e4m3, grid, s))
                   : (page == 64 ? fwd_launch_of<P, 128, 64>(p, rows, e4m3, grid, s) : fwd_launch_of<P, 128, 128>(p, rows, e4m3, grid, s));
}

// merge_rows: rows of a workgroup, one or as many as have a thread per 16 bytes
template <class P>
hipError_t merge_launch(const P& p, int tile_rows, int d, int page, unsigned grid, int merge_rows, hipStream_t s)
{
    auto merge = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, p, tile_rows, page); };
    if (d == 64)
        merge_rows == 1 ? merge(cache_merge<64, 16, P>) : merge(cache_merge<64, 1, P>);
    else
        merge_rows == 1 ? merge(cache_merge<128, 8, P>) : merge(cache_merge<128, 1, P>);
    return hipGetLastError();
}

}  // namespace

}  // namespace attn
