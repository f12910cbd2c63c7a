// Eviction: the tokens to keep of every (sequence, KV head), and their move into
// new pages.
//
// Choice: the k-th largest weight by its bits, eight at a time (a histogram of
// the weights that agree so far, in LDS), then one ordered pass that numbers the
// kept tokens.  One workgroup per (sequence, head): the passes read 4 bytes per
// token from L2 and are bound by their chain (four histograms, the ordered pass),
// not by memory.  Move: one workgroup per new block, head, and K or V gathers the
// block's rows into registers, takes their largest value and writes the codes.
#include "cache_common.hpp"

#include <type_traits>

namespace attn {

namespace {

constexpr int kPick = 1024;      // threads of a choosing workgroup

// Order of the weights as unsigned numbers: NaN lowest, -0 equal to 0.
__device__ inline uint32_t weight_key(float w)
{
    if (w != w)
        return 0u;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kPick) evict_pick(EvictParams p, int max_len)
{
    constexpr int NW = kPick / 64;
    __shared__ uint32_t hist[256];
    __shared__ uint32_t wsum[2][NW];
    __shared__ uint32_t found[2];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int hk = (int)(blockIdx.x % p.from.Hkv), b = (int)(blockIdx.x / p.from.Hkv);
    const int len = min(max(p.bt.lens[b], 0), max_len);
    const int m = min(len, p.budget);
    const float* const w = p.w + (int64_t)b * p.sb + (int64_t)hk * p.sh;
    const size_t row = ((size_t)b * p.from.Hkv + hk) * p.budget;
    int32_t* const kept = p.kept + row;
    float* const nw = p.new_w ? p.new_w + row : nullptr;
    if (hk == 0 && tid == 0)
        p.new_lens[b] = m;
    for (int i = m + tid; i < p.budget; i += kPick) {
        kept[i] = -1;
        if (nw)
            nw[i] = 0.f;
    }
    // [0, lo) and [hi, len) are kept, of [lo, hi) the `want` largest
    int lo = len, hi = len, want = 0;
    if (len > p.budget) {
        lo = min(p.n_sink, p.budget);
        const int recent = min(p.n_recent, p.budget - lo);
        hi = len - recent;
        want = p.budget - lo - recent;
    }
    // the key of the last one kept, and how many equal to it
    uint32_t key = 0;
    uint32_t left = (uint32_t)want;
    if (want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256)
                hist[tid] = 0u;
            __syncthreads();
            for (int t = lo + tid; t < hi; t += kPick) {
                const uint32_t k = weight_key(w[t]);
                if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8)))
                    atomicAdd(&hist[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            // from the top: the digit at which `left` are reached
            if (tid < 64) {
                uint32_t c[4], mine = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c[j] = hist[255 - (4 * lane + j)];
                    mine += c[j];
                }
                uint32_t before = mine;
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) {
                    const uint32_t t = (uint32_t)__shfl_up((int)before, off, 64);
                    if (lane >= off)
                        before += t;
                }
                before -= mine;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (before < left && before + c[j] >= left) {
                        found[0] = 255u - (4 * lane + j);
                        found[1] = left - before;
                    }
                    before += c[j];
                }
            }
            __syncthreads();
            key |= found[0] << shift;
            left = found[1];
            __syncthreads();
        }
    }
    // number the kept ones in order
    uint32_t base = 0, equal = 0;
    for (int t0 = 0; t0 < len; t0 += kPick) {
        const int t = t0 + tid;
        const bool in = t < len, middle = in && t >= lo && t < hi;
        const float x = in ? w[t] : 0.f;
        const uint32_t k = weight_key(x);
        const bool eq = middle && want > 0 && k == key;
        const uint64_t eqs = __ballot(eq);
        if (lane == 0)
            wsum[0][wv] = (uint32_t)__popcll(eqs);
        __syncthreads();
        uint32_t eb = equal;
        for (int i = 0; i < NW; ++i) {
            const uint32_t c = wsum[0][i];
            eb += i < wv ? c : 0u;
            equal += c;
        }
        const uint64_t below = (1ull << lane) - 1;
        const uint32_t erank = eb + (uint32_t)__popcll(eqs & below);
        const bool keep = in && (!middle || (want > 0 && (k > key || (eq && erank < left))));
        const uint64_t ks = __ballot(keep);
        if (lane == 0)
            wsum[1][wv] = (uint32_t)__popcll(ks);
        __syncthreads();
        uint32_t kb = base;
        for (int i = 0; i < NW; ++i) {
            const uint32_t c = wsum[1][i];
            kb += i < wv ? c : 0u;
            base += c;
        }
        const uint32_t at = kb + (uint32_t)__popcll(ks & below);
        if (keep && at < (uint32_t)m) {
            kept[at] = t;
            if (nw)
                nw[at] = x;
        }
    }
}

template <int D, int PAGE>
__global__ void __launch_bounds__(256) evict_move(EvictParams p)
{
    constexpr int UPT = D / 16, TPP = 256 / UPT, NP = PAGE / TPP;
    int64_t i = blockIdx.x;
    const bool is_v = i & 1;
    i >>= 1;
    const int hk = (int)(i % p.from.Hkv);
    i /= p.from.Hkv;
    const int block = (int)(i % p.nb), b = (int)(i / p.nb);
    const int m = min(min(max(p.bt.lens[b], 0), p.bt.W * PAGE), p.budget);
    const int z = min(m - block * PAGE, PAGE);      // tokens of the block
    if (z <= 0)
        return;
    const int pid = p.new_pages[(size_t)b * p.nb + block];
    if ((uint32_t)pid >= (uint32_t)p.to.n_pages)
        return;
    const int32_t* const kept = p.kept + ((size_t)b * p.from.Hkv + hk) * p.budget + block * PAGE;
    const uint8_t* const src = is_v ? p.from.v : p.from.k;
    const uint8_t* const src_scale = is_v ? p.from.vs : p.from.ks;
    const int u = threadIdx.x % UPT, tk = threadIdx.x / UPT;
    i32x4 code[NP];
    int ex[NP];
    float amax = 0.f;
#pragma unroll
    for (int q = 0; q < NP; ++q) {
        const int slot = q * TPP + tk;
        code[q] = i32x4{};
        ex[q] = 0;
        if (slot >= z)
            continue;
        const int t = kept[slot];
        const int from = t < 0 ? -1 : page_of(p.bt, p.from.n_pages, b, t / PAGE);
        if (from < 0)
            continue;                               // (no page: zeros)
        const size_t at = (size_t)from * p.from.Hkv + hk;
        code[q] = *reinterpret_cast<const i32x4*>(src + at * (PAGE * D) + (t % PAGE) * D + 16 * u);
        ex[q] = (int)src_scale[at] - 127;
        float top = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float y[4];
            from_e4m3((uint32_t)code[q][c], y);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top = fmax_f(top, __builtin_fabsf(y[e]));   // (a NaN code does not count)
        }
        amax = fmax_f(amax, __builtin_amdgcn_ldexpf(top, ex[q]));
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        amax = fmax_f(amax, __shfl_xor(amax, off, 64));
    __shared__ float wave_max[4];
    if ((threadIdx.x & 63) == 0)
        wave_max[threadIdx.x >> 6] = amax;
    __syncthreads();
    amax = fmax_f(fmax_f(wave_max[0], wave_max[1]), fmax_f(wave_max[2], wave_max[3]));
    const int e = block_exponent(amax);
    const size_t to = (size_t)pid * p.to.Hkv + hk;
    uint8_t* const dst = (is_v ? p.to.v : p.to.k) + to * (PAGE * D);
    if (threadIdx.x == 0)
        (is_v ? p.to.vs : p.to.ks)[to] = (uint8_t)(e + 127);
#pragma unroll
    for (int q = 0; q < NP; ++q) {
        const int slot = q * TPP + tk;
        if (slot >= z)
            continue;
        i32x4 x = code[q];
        if (ex[q] != e) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float y[4];
                from_e4m3((uint32_t)x[c], y);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    y[k] = __builtin_amdgcn_ldexpf(y[k], ex[q] - e);
                x[c] = (int)to_e4m3(y[0], y[1], y[2], y[3]);
            }
        }
        *reinterpret_cast<i32x4*>(dst + slot * D + 16 * u) = x;
    }
}

}  // namespace

hipError_t launch_cache_evict(const EvictParams& p, int d, int page, hipStream_t s)
{
    const int64_t heads = (int64_t)p.bt.B * p.from.Hkv, moves = heads * p.nb * 2;
    if (moves > 1 << 30)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(evict_pick, dim3((unsigned)heads), dim3(kPick), 0, s, p, p.bt.W * page);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)moves), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    if (d == 64)
        return page == 64 ? go(evict_move<64, 64>) : go(evict_move<64, 128>);
    return page == 64 ? go(evict_move<128, 64>) : go(evict_move<128, 128>);
}

}  // namespace attn
