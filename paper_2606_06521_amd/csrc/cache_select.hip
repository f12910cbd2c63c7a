// Choice of pages: for a run of new tokens and a KV head the pages whose bounds allow the
// largest scores.
//
// A key k of a page lies between lo and hi in every channel, so q k <= sum_c max(q lo, q hi)
// = q+ hi + q- lo with q+ and q- the positive and negative parts of q: two matrix products.
// q is rounded to whole numbers up to 127 on a power of two of its row, lo and hi are codes
// that are multiples of 1/2 up to 448: sums of 128 channels stay below 2^24 of these halves,
// so the bf16 matrix cores' FP32 sums are exact in any order and the choice does not depend on it.
//
// One workgroup per list.  A wave takes every NW-th 32 pages: S = Q B^T in tiles of 32 rows
// by 32 pages, lane n holding 16 rows' scores of page n, so that a page's largest is taken
// within the lane.  Keys that order as the scores do then go through a radix choice in LDS.
#include "cache_common.hpp"

namespace attn {

namespace {

// Orders as the numbers do, as unsigned; above 0 and below the largest.
__device__ inline uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// What the wave's lanes wrote to LDS is read by its others.
__device__ inline void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int D, bool E4M3, int NW, int MOST>
__global__ void __launch_bounds__(64 * NW) select_kernel(SelectParams p, int page)
{
    constexpr int NI = D / 32;              // 16-byte pieces of a row and half
    __shared__ float score[MOST];
    __shared__ int row_e[NW][32], row_last[NW][32];
    __shared__ int hist[256], wave_sum[NW + 1][2];

    const int units = p.bt.B * p.cache.Hkv * p.runs, per_xcd = (units + kNumXcd - 1) / kNumXcd;
    const int slot = (int)(blockIdx.x / kNumXcd), unit = (int)(blockIdx.x % kNumXcd) * per_xcd + slot;
    if (slot >= per_xcd || unit >= units)
        return;
    const int run = unit % p.runs, hk = unit / p.runs % p.cache.Hkv, b = unit / p.runs / p.cache.Hkv;
    Seq s = uniform(sequence(p.bt, b, p.max_len));
    s.first += run * p.run;
    s.pos0 += run * p.run;
    s.n = min(max(s.n - run * p.run, 0), p.run);
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const int rows = s.n * p.gr.G;
    const int seen = s.n > 0 ? last_key(s.pos0 + s.n - 1, p.causal, s.len) + 1 : 0;
    const int nb = (max(seen, 0) + page - 1) / page;
    int32_t* const list = p.blocks + (((int64_t)b * p.runs + run) * p.cache.Hkv + hk) * p.take;

    // ---- scores ----
    for (int row0 = 0; row0 < rows; row0 += 32) {
        bf16x8 qp[2 * NI], qn[2 * NI];
        {
            const int row = min(row0 + n, rows - 1), i = p.gr.token(row);
            const int64_t at = (int64_t)(s.first + i) * p.q.st + (int64_t)(hk * p.gr.G + (row - i * p.gr.G)) * p.q.sh;
            typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
            u16x8 m = {};
#pragma unroll
            for (int j = 0; j < 2 * NI; ++j) {
                qp[j] = load_q8<E4M3>(p.q.data, at + 32 * (j / 2) + 16 * h + 8 * (j % 2));
                m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x8, qp[j]) & (u16x8)((uint16_t)0x7FFF));
            }
            uint16_t top = 0;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                top = m[c] > top ? m[c] : top;
            top = (uint16_t)max((int)top, __shfl_xor((int)top, 32, 64));
            const bool good = top < 0x7F80;
            const float f = __uint_as_float((uint32_t)top << 16);
            // least e with f <= 127 2^e: 127 = 0.9921875 * 2^7
            const int e = __builtin_amdgcn_frexp_expf(f) - 7 + (__builtin_amdgcn_frexp_mantf(f) > 0.9921875f ? 1 : 0);
#pragma unroll
            for (int j = 0; j < 2 * NI; ++j)
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float x = good ? __builtin_rintf(__builtin_amdgcn_ldexpf((float)qp[j][c], -e)) : 0.f;
                    qp[j][c] = (__bf16)fmax_f(x, 0.f);
                    qn[j][c] = (__bf16)-fmax_f(-x, 0.f);
                }
            if (h == 0) {
                row_e[w][n] = e;
                // (a row that is not finite, or none, sees no page)
                row_last[w][n] = good && row0 + n < rows ? last_key(s.pos0 + i, p.causal, s.len) : -1;
            }
        }
        wave_fence();
        for (int b0 = 32 * w; b0 < nb; b0 += 32 * NW) {
            const int block = b0 + n;
            const int pid = block < nb ? page_of(p.bt, p.cache.n_pages, b, block) : -1;
            const size_t at = (size_t)max(pid, 0) * p.cache.Hkv + hk;
            i32x4 x[2][NI];
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int i = 0; i < NI; ++i)
                    x[part][i] = pid < 0 ? i32x4{}
                                         : *reinterpret_cast<const i32x4*>(p.bounds + at * (2 * D) + part * D + 32 * i + 16 * h);
            const int kb = pid < 0 ? 0 : p.cache.ks[at] - 127;
            f32x16 acc = {};
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const i32x4 v = x[part][i];
                    const bf16x8 k0 = widen((uint32_t)v[0], (uint32_t)v[1]), k1 = widen((uint32_t)v[2], (uint32_t)v[3]);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part ? qp[2 * i] : qn[2 * i], k0, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(part ? qp[2 * i + 1] : qn[2 * i + 1], k1, acc, 0, 0, 0);
                }
            float best = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = 8 * (r / 4) + 4 * h + r % 4;
                const int up = min(max(row_e[w][row] + kb, -96), 96);
                const float u = __builtin_amdgcn_ldexpf(acc[r], up);
                best = fmax_f(best, block * page <= row_last[w][row] ? u : -INFINITY);
            }
            best = halves_max(best);
            if (h == 0 && block < nb) {
                if (row0 > 0)
                    best = fmax_f(best, score[block]);
                // (the last rows: as a key)
                if (row0 + 32 >= rows)
                    best = __uint_as_float(pid < 0 ? 0u : block < p.n_first || block >= nb - p.n_last ? ~0u : key_of(best));
                score[block] = best;
            }
        }
        wave_fence();
    }
    __syncthreads();
    const uint32_t* const key = reinterpret_cast<const uint32_t*>(score);

    // ---- the key of the last page taken, and how many of its equals are ----
    // radix choice, eight bits a round from the top: the pages above `floor` are in, `left` of
    // those that share its bits so far are still to be found
    uint32_t floor = 0;
    int left = p.take;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += 64 * NW)
            hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < nb; i += 64 * NW) {
            const uint32_t k = key[i];
            if (shift == 24 || k >> (shift + 8) == floor >> (shift + 8))
                atomicAdd(&hist[k >> shift & 255], 1);
        }
        __syncthreads();
        // the highest digit with `left` pages at or above it (0 if there are fewer)
        if (w == 0) {
            int c[4], sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = hist[255 - (4 * lane + j)];
                sum += c[j];
            }
            int before = sum;
#pragma unroll
            for (int off = 1; off < 64; off *= 2) {
                const int o = __shfl_up(before, off, 64);
                before += lane >= off ? o : 0;
            }
            before -= sum;
            int digit = -1, above = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (digit < 0 && before < left && before + c[j] >= left) {
                    digit = 255 - (4 * lane + j);
                    above = before;
                }
                before += c[j];
            }
            const uint64_t who = __ballot(digit >= 0);
            if (who == 0 ? lane == 0 : lane == __builtin_ctzll(who)) {
                wave_sum[NW][0] = who == 0 ? -1 : digit;
                wave_sum[NW][1] = above;
            }
        }
        __syncthreads();
        const int digit = wave_sum[NW][0];
        if (digit < 0) {        // fewer pages than the list takes: all
            floor = 0;
            left = 0;
            break;
        }
        floor |= (uint32_t)digit << shift;
        left -= wave_sum[NW][1];
    }
    // (a page that is none has the key 0 and is not taken)
    if (floor == 0)
        left = 0;

    // ---- their places, in order: a wave's part of the pages ----
    const int per_wave = (nb + 64 * NW - 1) / (64 * NW) * 64, i0 = w * per_wave, i1 = min(i0 + per_wave, nb);
    int above = 0, equal = 0;
    for (int i = i0; i < i1; i += 64) {
        const uint32_t k = i + lane < i1 ? key[i + lane] : 0u;
        above += __builtin_popcountll(__ballot(k > floor));
        equal += __builtin_popcountll(__ballot(k == floor && floor != 0));
    }
    __syncthreads();
    if (lane == 0) {
        wave_sum[w][0] = above;
        wave_sum[w][1] = equal;
    }
    __syncthreads();
    int sure = 0, ties = 0, all = 0, all_ties = 0;
    for (int i = 0; i < NW; ++i) {
        sure += i < w ? wave_sum[i][0] : 0;
        ties += i < w ? wave_sum[i][1] : 0;
        all += wave_sum[i][0];
        all_ties += wave_sum[i][1];
    }
    for (int i = i0; i < i1; i += 64) {
        const uint32_t k = i + lane < i1 ? key[i + lane] : 0u;
        const uint64_t hi = __ballot(k > floor), eq = __ballot(k == floor && floor != 0), below = ((uint64_t)1 << lane) - 1;
        const int t = ties + __builtin_popcountll(eq & below);
        const bool in = k > floor || (eq >> lane & 1 && t < left);
        if (in)
            list[sure + __builtin_popcountll(hi & below) + min(t, left)] = i + lane;
        sure += __builtin_popcountll(hi);
        ties += __builtin_popcountll(eq);
    }
    for (int i = all + min(all_ties, left) + tid; i < p.take; i += 64 * NW)
        list[i] = -1;
}

}  // namespace

hipError_t launch_cache_select(const SelectParams& p, int d, int page, bool e4m3, hipStream_t s)
{
    const __int128 units = (__int128)p.bt.B * p.cache.Hkv * p.runs;
    unsigned grid;
    const hipError_t e = grid_of((units + kNumXcd - 1) / kNumXcd * kNumXcd, 256, grid);
    if (e != hipSuccess)
        return e;
    auto go = [&](auto kern, int nw) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * nw), 0, s, p, page);
        return hipGetLastError();
    };
    if (d == 64)
        return e4m3 ? go(select_kernel<64, true, 4, kMaxChoice>, 4) : go(select_kernel<64, false, 4, kMaxChoice>, 4);
    return e4m3 ? go(select_kernel<128, true, 4, kMaxChoice>, 4) : go(select_kernel<128, false, 4, kMaxChoice>, 4);
}

}  // namespace attn
