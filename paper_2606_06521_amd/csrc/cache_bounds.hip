// Bounds of a page's keys: of each channel the least and the largest code, rounded outwards
// to a multiple of 1/2.
//
// One workgroup per page and KV head reads its codes once, 16 bytes a thread and row.  Codes
// are compared as signed bytes, in the upper halves of 16-bit numbers (a negative code's
// magnitude is complemented, which orders them), two to an instruction.
// What bounds it: single tokens the chain of loads (length, page, K) and the launch, 4.1 us for
// 16 sequences; prompts of 22.6 MB of K (4 x 8 heads, up to 8192 keys, d = 128) 9.1 to 10.2 us, the same
// chain and then 4 us of the stream: all workgroups start at once and each has its whole page on the way.
#include "cache_common.hpp"

#include <algorithm>

namespace attn {

namespace {

typedef int16_t s16x2_t __attribute__((ext_vector_type(2)));

// The codes of a word as signed bytes of the same order (it is its own inverse).
__device__ inline uint32_t ordered(uint32_t w) { return w ^ (((w >> 7) & 0x01010101u) * 0x7Fu); }

// Bounds of page `block` of sequence b, of its keys before `to`; by all threads of the workgroup.
template <int D, int PAGE>
__device__ inline void page_bounds(const BoundsParams& p, int b, int hk, int block, int to, int (&lo_sh)[4][D / 2], int (&hi_sh)[4][D / 2])
{
    constexpr int CPR = D / 16, RPP = 256 / CPR, NL = (PAGE + RPP - 1) / RPP;       // chunks of a row, rows of a pass
    const int pid = __builtin_amdgcn_readfirstlane(page_of(p.bt, p.cache.n_pages, b, block));
    if (pid < 0)
        return;
    // (tokens behind the new ones are not of this call, those before them are in the page)
    const int count = min(to - block * PAGE, PAGE);
    const size_t at = (size_t)pid * p.cache.Hkv + hk;
    const uint8_t* const page = p.cache.k + at * ((size_t)PAGE * D);

    const int tid = threadIdx.x, c = tid % CPR, r0 = tid / CPR;
    i32x4 x[NL];
#pragma unroll
    for (int l = 0; l < NL; ++l)
        // (a row past the count reads the first, and counts for nothing new)
        x[l] = *reinterpret_cast<const i32x4*>(page + (r0 + l * RPP < count ? r0 + l * RPP : 0) * D + 16 * c);
    s16x2_t lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo[i] = s16x2_t{32767, 32767};
        hi[i] = s16x2_t{-32768, -32768};
    }
#pragma unroll
    for (int l = 0; l < NL; ++l)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t w = (uint32_t)x[l][j];
            w = ordered(w & ~((nan_bytes(w) >> 7) * 255u));
            const s16x2_t half[2] = {__builtin_bit_cast(s16x2_t, (w << 8) & 0xFF00FF00u), __builtin_bit_cast(s16x2_t, w & 0xFF00FF00u)};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                lo[2 * j + e] = __builtin_elementwise_min(lo[2 * j + e], half[e]);
                hi[2 * j + e] = __builtin_elementwise_max(hi[2 * j + e], half[e]);
            }
        }
    const int lane = tid & 63, w = tid >> 6;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int off = CPR; off < 64; off *= 2) {
            lo[i] = __builtin_elementwise_min(lo[i], __builtin_bit_cast(s16x2_t, __shfl_xor(__builtin_bit_cast(int, lo[i]), off, 64)));
            hi[i] = __builtin_elementwise_max(hi[i], __builtin_bit_cast(s16x2_t, __shfl_xor(__builtin_bit_cast(int, hi[i]), off, 64)));
        }
        if (lane < CPR) {
            lo_sh[w][8 * c + i] = __builtin_bit_cast(int, lo[i]);
            hi_sh[w][8 * c + i] = __builtin_bit_cast(int, hi[i]);
        }
    }
    __syncthreads();
    // four channels a thread: words 2 j (bytes 0 and 2) and 2 j + 1 (bytes 1 and 3) of either bound
    if (tid < D / 2) {
        const bool upper = tid >= D / 4;
        const int j = upper ? tid - D / 4 : tid;
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            s16x2_t v = __builtin_bit_cast(s16x2_t, upper ? hi_sh[0][2 * j + e] : lo_sh[0][2 * j + e]);
#pragma unroll
            for (int i = 1; i < 4; ++i) {
                const s16x2_t o = __builtin_bit_cast(s16x2_t, upper ? hi_sh[i][2 * j + e] : lo_sh[i][2 * j + e]);
                v = upper ? __builtin_elementwise_max(v, o) : __builtin_elementwise_min(v, o);
            }
            word |= e ? __builtin_bit_cast(uint32_t, v) : __builtin_bit_cast(uint32_t, v) >> 8;
        }
        float f[4];
        from_e4m3(ordered(word), f);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            // (a multiple of 1/2 below 4 has three bits, any code from 4 on is one; -0 becomes 0)
            f[i] = (upper ? __builtin_ceilf(2.f * f[i]) : __builtin_floorf(2.f * f[i])) * 0.5f + 0.f;
        *reinterpret_cast<uint32_t*>(p.bounds + at * (2 * D) + (upper ? D : 0) + 4 * j) = to_e4m3(f[0], f[1], f[2], f[3]);
    }
}

template <int D, int PAGE>
__global__ void __launch_bounds__(256) bounds_kernel(BoundsParams p)
{
    __shared__ int lo_sh[4][D / 2], hi_sh[4][D / 2];
    const int hk = (int)(blockIdx.x % p.cache.Hkv);
    const int rest = (int)(blockIdx.x / p.cache.Hkv);
    const int b = rest / p.step;
    const Seq s = uniform(sequence(p.bt, b, p.bt.W * PAGE));
    const int from = max(s.pos0, 0), to = min(s.pos0 + s.n, s.len);
    if (from >= to)
        return;
    for (int block = from / PAGE + rest % p.step; block * PAGE < to; block += p.step) {
        page_bounds<D, PAGE>(p, b, hk, block, to, lo_sh, hi_sh);
        if ((block + p.step) * PAGE < to)
            __syncthreads();            // (the next page's bounds go to the same LDS)
    }
}

}  // namespace

// (most: pages of a sequence that may hold new tokens)
hipError_t launch_cache_bounds(BoundsParams p, int most, int d, int page, hipStream_t s)
{
    // One workgroup per page and head.  Tables with room for more than a launch has workgroups for hold
    // far fewer tokens: 2^20 workgroups then take the pages that there are in turns.
    const int64_t heads = (int64_t)p.bt.B * p.cache.Hkv;
    unsigned grid;
    p.step = most;
    if (grid_of((__int128)heads * most, 256, grid) != hipSuccess)
        p.step = (int)std::max<int64_t>((1 << 20) / heads, 1);
    const hipError_t e = grid_of((__int128)heads * p.step, 256, grid);
    if (e != hipSuccess)
        return e;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    return d == 64 ? (page == 64 ? go(bounds_kernel<64, 64>) : go(bounds_kernel<64, 128>))
                   : (page == 64 ? go(bounds_kernel<128, 64>) : go(bounds_kernel<128, 128>));
}

}  // namespace attn
