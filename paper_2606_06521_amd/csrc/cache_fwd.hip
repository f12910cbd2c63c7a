// Attention of new tokens over the cache: plan, launch, merge.
#include "cache_fwd_tile.hpp"

#include <algorithm>
#include <type_traits>

namespace attn {

namespace {

// Ranges of a tile at most: 2^26 keys in ranges of kMaxChunk visits.
constexpr int kMergeRanges = 4096;
static_assert((1 << 26) / kVisit / kMaxChunk <= kMergeRanges && kTileChunk >= kMaxChunk);

// Merge of a split tile: a workgroup per query row, thread (piece, part) takes
// one 16-byte piece of the row from every PARTS-th range; the parts are added
// through LDS in a fixed order.  Ranges stand at their own power of two; the
// row's is the largest.
template <int D>
__global__ void __launch_bounds__(256) cache_merge(FwdParams p, int tile_rows)
{
    constexpr int PIECES = D / 4, PARTS = 256 / PIECES;
    __shared__ f32x4 osh[PARTS][PIECES];
    __shared__ float lsh[PARTS], msh[kMergeRanges], wave_max[4];
    const int hk = (int)(blockIdx.x % p.cache.Hkv);
    int64_t rest = blockIdx.x / p.cache.Hkv;
    const int per_seq = p.bt.max_q * p.gr.G;
    const int b = (int)(rest / per_seq), R = (int)(rest - (int64_t)b * per_seq);
    const Seq s = sequence(p.bt, b, p.max_len);
    if (R >= s.n * p.gr.G)
        return;
    const int tile = R / tile_rows;
    const int visits = tile_visits(p, s, tile, tile_rows);
    const int n = (visits + p.chunk - 1) / p.chunk;
    if (n <= 1)
        return;                                  // (the range wrote the row itself)
    const int rr = R - tile * tile_rows;
    const size_t stride = (size_t)tile_rows * (D + 2);
    const float* base = p.ws + (((size_t)b * p.cache.Hkv + hk) * p.tiles + tile) * p.ranges * stride;
    const int piece = threadIdx.x % PIECES, part = threadIdx.x / PIECES;
    // the ranges' references, all loaded at once
    float m = -INFINITY;
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
    f32x4 acc = {};
    float l = 0.f;
#pragma unroll 4
    for (int c = part; c < n; c += PARTS) {
        const float* at = base + c * stride;
        const f32x4 x = *reinterpret_cast<const f32x4*>(at + rr * D + 4 * piece);
        const float lc = at[tile_rows * D + rr], mc = msh[c];
        const float f = mc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - m);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc[e] += x[e] * f;
        l += lc * f;
    }
    osh[part][piece] = acc;
    if (piece == 0)
        lsh[part] = l;
    __syncthreads();
    if (part != 0)
        return;
#pragma unroll
    for (int v = 1; v < PARTS; ++v) {
        const f32x4 t = osh[v][piece];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc[e] += t[e];
        l += lsh[v];
    }
    write_row<D>(p, s, hk, R, piece, acc, l, 1.f / l, m);
}

template <int D, int PAGE>
hipError_t fwd_go(const FwdParams& p, int rows, bool e4m3, int64_t grid, hipStream_t s)
{
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    if (rows == kTileRows)
        return e4m3 ? go(cache_fwd_tile_kernel<D, PAGE, true>) : go(cache_fwd_tile_kernel<D, PAGE, false>);
    return e4m3 ? go(cache_fwd_kernel<D, PAGE, true>) : go(cache_fwd_kernel<D, PAGE, false>);
}

// Query rows of a (sequence, KV head) beyond which tiles of 128 rows take less time
// than tiles of 16, each of which streams K and V by itself.
constexpr int kTallFrom = 32;

}  // namespace

FwdPlan cache_fwd_plan(int B, int Hkv, int G, int max_q, int max_len, int d, int n_cu)
{
    FwdPlan pl;
    const int64_t run = (int64_t)max_q * G;             // rows of a (sequence, KV head)
    const bool tall = run > kTallFrom;
    pl.rows = tall ? kTileRows : 16;
    pl.tiles = (int)((run + pl.rows - 1) / pl.rows);
    const int64_t units = (int64_t)B * Hkv * pl.tiles;
    const int visits = (max_len + kVisit - 1) / kVisit;
    // enough ranges to fill the GPU (two workgroups of tall tiles fit a CU), none
    // shorter than two visits of a workgroup's four waves, or eight of a tall tile's
    const int64_t want = std::min<int64_t>(std::max<int64_t>(1, (tall ? 2 : 1) * n_cu / std::max<int64_t>(units, 1)), kMergeRanges);
    pl.chunk = (int)std::max<int64_t>(8, (visits + want - 1) / want);
    pl.chunk = std::min(pl.chunk, tall ? kTileChunk : kMaxChunk);
    pl.ranges = std::max(1, (visits + pl.chunk - 1) / pl.chunk);
    pl.bytes = pl.ranges > 1 ? (size_t)units * pl.ranges * pl.rows * (d + 2) * sizeof(float) : 0;
    return pl;
}

hipError_t launch_cache_fwd(FwdParams p, const FwdPlan& pl, int d, int page, bool e4m3, hipStream_t s)
{
    p.tiles = pl.tiles;
    p.chunk = pl.chunk;
    p.ranges = pl.ranges;
    const int64_t units = (int64_t)p.bt.B * p.cache.Hkv * pl.tiles;
    // (whole rounds of the XCDs)
    const int64_t grid = (units * pl.ranges + kNumXcd - 1) / kNumXcd * kNumXcd, rows = (int64_t)p.bt.B * p.cache.Hkv * p.bt.max_q * p.gr.G;
    if (grid > 1 << 30 || rows > 1 << 30)
        return hipErrorInvalidValue;
    hipError_t e = d == 64 ? (page == 64 ? fwd_go<64, 64>(p, pl.rows, e4m3, grid, s) : fwd_go<64, 128>(p, pl.rows, e4m3, grid, s))
                           : (page == 64 ? fwd_go<128, 64>(p, pl.rows, e4m3, grid, s) : fwd_go<128, 128>(p, pl.rows, e4m3, grid, s));
    if (e == hipSuccess && pl.ranges > 1) {
        if (d == 64)
            hipLaunchKernelGGL(cache_merge<64>, dim3((unsigned)rows), dim3(256), 0, s, p, pl.rows);
        else
            hipLaunchKernelGGL(cache_merge<128>, dim3((unsigned)rows), dim3(256), 0, s, p, pl.rows);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace attn
