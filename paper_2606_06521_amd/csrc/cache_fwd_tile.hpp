// Attention over the cache: tiles of 128 query rows (chunks of a prompt).
//
// The rows of a (sequence, KV head) as in cache_fwd_kernel.hpp, four waves of 32
// of them; the waves share each visit's K and V in LDS, double-buffered, every
// wave loading a quarter, one barrier per visit.  Two workgroups fit a CU: one's
// matrix work can run beside the other's softmax.
//
// S^T by the 32x32x16 bf16 MFMA: its tile of 32 keys is a group of P, the lane of
// row n and half h holds its keys 16 h .. 16 h + 15, and the pair's E4M3 bytes
// are the operand of the 32x32x64 E4M3 MFMA of P.V.  The group's power of two,
// the row's reference and V's scale are as there.
//
// What bounds it is vector work: per key and row an exp2 (half of the rate), an FMA,
// an add, half a maximum and half a convert, and the widening of K's codes to bf16,
// which 32 rows share: 76 % of the cycles, beside 44 % of the matrix cores'.
// 8 heads x 2048 x 4 rows against 16384 keys, d = 128: 396 to 408 us, by the card, 1.26 to 1.30
// PFLOP/s; a large bf16 product reaches 1.40.  Q comes through LDS in whole lines (gathered from memory by
// the lanes that use it, each line is read 8 times).
#pragma once

#include "cache_fwd_kernel.hpp"

#include <algorithm>

namespace attn {

// The lane's number, anew: kept through the loop it would go to scratch memory, and the waits for
// K and V would wait for that too (5 us of a short range's 30).
__device__ inline int lane_now()
{
    uint32_t zero = 0;
    asm volatile("" : "+s"(zero));
    return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

constexpr int kTileRows = 128;
constexpr int kTileChunk = 512;     // visits of a range

template <int D, int PAGE, class P>
struct TallLds {
    static constexpr int kStage = 4 * kVisit * D, kPages = kTileChunk * (kVisit / PAGE);
    uint8_t* lds;                   // kStage bytes, 1024-byte aligned: K, V, K, V
    int* pids;                      // kPages
    uint8_t *kbyte, *vbyte;         // kPages
    int* starts;                    // lists: kPages, first keys of the pages
    int* row_last;                  // shared pages: kTileRows
};

template <int D, int PAGE, bool E4M3, class P>
__global__ void __launch_bounds__(256, 2) cache_fwd_tile_kernel(P p)
{
    using Lds = TallLds<D, PAGE, P>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[Lds::kStage];
    __shared__ int pids[Lds::kPages];
    __shared__ uint8_t kbyte[Lds::kPages], vbyte[Lds::kPages];
    __shared__ int starts[kLists<P> ? Lds::kPages : 1], row_last[kShared<P> ? kTileRows : 1];
#include "cache_fwd_tall.inc"
}

// The same as a part of another kernel.
template <int D, int PAGE, bool E4M3, class P>
__device__ __forceinline__ void tall_tile(const P& p, const TallLds<D, PAGE, P>& sh)
{
    uint8_t* const lds = sh.lds;
    int *const pids = sh.pids, *const starts = sh.starts, *const row_last = sh.row_last;
    uint8_t *const kbyte = sh.kbyte, *const vbyte = sh.vbyte;
#include "cache_fwd_tall.inc"
}

// The shared pages on 128-row tiles and, in the workgroups behind theirs, the sequences' own on 16-row
// tiles.  Two workgroups fit a CU: the two kinds wait for memory at different times.
template <int D, int PAGE, bool E4M3>
__global__ void __launch_bounds__(256, 2) cache_fwd_both_kernel(SharedParams p)
{
    constexpr int STAGES = D == 64 ? 2 : 1;
    using Tall = TallLds<D, PAGE, SharedParams>;
    using Low = LowLds<D, PAGE, SharedParams, STAGES>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[std::max(Tall::kStage, Low::kStage)];
    __shared__ int pids[std::max(Tall::kPages, Low::kPages)];
    __shared__ uint8_t kbyte[std::max(Tall::kPages, Low::kPages)], vbyte[std::max(Tall::kPages, Low::kPages)];
    __shared__ float lsh[4][16], msh[4][16];
    __shared__ int row_last[kTileRows];
    if (blockIdx.x < p.pre_grid)
        tall_tile<D, PAGE, E4M3, SharedParams>(p, {lds, pids, kbyte, vbyte, nullptr, row_last});
    else
        low_tile<D, PAGE, E4M3, SharedParams, STAGES>(p, {lds, pids, kbyte, vbyte, lsh, msh, nullptr, row_last});
}

}  // namespace attn
