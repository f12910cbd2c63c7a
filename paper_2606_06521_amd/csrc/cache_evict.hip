// Eviction: the tokens to keep of every (sequence, KV head), and their move into
// new pages.
//
// Choice: the k-th largest weight by its bits, eleven at a time (a histogram of
// the weights that agree so far, in LDS), then the kept tokens are numbered in
// their order.  One workgroup per (sequence, head), which keeps up to 16384
// weights in registers: bound by the chain of rounds, not by memory (4096 tokens 7.6
// us, 8192 11).  Move: one workgroup per new block, head, and K or V gathers the
// block's rows into registers, takes their largest value and writes the codes: rows of
// 128 bytes at random, 16 x 8 heads x 2048 tokens in 30 us, 3.6 TB/s read and written.
#include "cache_common.hpp"

#include <type_traits>

namespace attn {

namespace {

constexpr int kPick = 1024;      // threads of a choosing workgroup
constexpr int kDigit = 11;       // bits per round of the choice: 11, 11, 10

// Order of the weights as unsigned numbers: NaN lowest, -0 equal to 0.
__device__ inline uint32_t weight_key(float w)
{
    if (w != w)
        return 0u;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// Inclusive sum over the lanes of a wave, by lane shifts within rows of 16 and two
// broadcasts of a row's last lane (a tenth of the time of shuffles through LDS).
__device__ inline uint32_t wave_scan(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);
    return x;
}

// E > 0: a thread keeps its E keys in registers (up to 1024 E tokens); E = 0: any
// number, read again in every round.
template <int E>
__global__ void __launch_bounds__(kPick) evict_pick(EvictParams p, int max_len)
{
    constexpr int NW = kPick / 64, BINS = 1 << kDigit, CAP = E > 0 ? E : 1;
    __shared__ uint32_t hist[BINS];
    __shared__ __attribute__((aligned(16))) uint32_t wsum[NW];
    __shared__ uint32_t found[2];
    __shared__ uint32_t tally[CAP * NW];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int hk = (int)(blockIdx.x % p.from.Hkv), b = (int)(blockIdx.x / p.from.Hkv);
    const float* const w = p.w + (int64_t)b * p.sb + (int64_t)hk * p.sh;
    const int len = min(max(p.bt.lens[b], 0), max_len);
    const int m = min(len, p.budget);
    const size_t row = ((size_t)b * p.from.Hkv + hk) * p.budget;
    int32_t* const kept = p.kept + row;
    float* const nw = p.new_w ? p.new_w + row : nullptr;
    float x[CAP];
    if constexpr (E > 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int t = e * kPick + tid;
            x[e] = t < len ? w[t] : 0.f;
        }
    }
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
    uint32_t key = 0, left = (uint32_t)want;
    if (want > 0) {
#pragma unroll
        for (int round = 0; round < 3; ++round) {
            const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, above = round == 1 ? 21 : 10;
            const uint32_t mask = round == 2 ? 1023u : BINS - 1;
            hist[tid] = 0u;
            hist[tid + kPick] = 0u;
            __syncthreads();
            auto count = [&](int t, float xt) __attribute__((always_inline)) {
                const uint32_t k = weight_key(xt);
                if (t >= lo && t < hi && (round == 0 || (k >> above) == (key >> above)))
                    atomicAdd(&hist[(k >> shift) & mask], 1u);
            };
            if constexpr (E > 0) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    count(e * kPick + tid, x[e]);
            } else {
                for (int t = lo + tid; t < hi; t += kPick)
                    count(t, w[t]);
            }
            __syncthreads();
            // from the top: the digit at which `left` are reached (two digits a thread)
            const int top = BINS - 1 - 2 * tid;
            const uint32_t c0 = hist[top], c1 = hist[top - 1];
            const uint32_t sum = wave_scan(c0 + c1);
            if (lane == 63)
                wsum[wv] = sum;
            __syncthreads();
            uint32_t before = sum - (c0 + c1);
#pragma unroll
            for (int i = 0; i < NW; ++i)
                before += i < wv ? wsum[i] : 0u;
            if (before < left && before + c0 + c1 >= left) {
                const bool second = before + c0 < left;
                found[0] = (uint32_t)(second ? top - 1 : top);
                found[1] = left - before - (second ? c0 : 0u);
            }
            __syncthreads();
            key |= found[0] << shift;
            left = found[1];
        }
    }
    const uint64_t below = (1ull << lane) - 1;
    auto put = [&](int t, float xt, uint32_t at) __attribute__((always_inline)) {
        if (at < (uint32_t)m) {
            kept[at] = t;
            if (nw)
                nw[at] = xt;
        }
    };
    if constexpr (E > 0) {
        // per run of 64 tokens (e, wave) the number of equal ones, then of kept ones;
        // their sums over the runs before it
        auto scan = [&]() __attribute__((always_inline)) {
            __syncthreads();
            if (wv == 0) {
                uint32_t base = 0;
#pragma unroll
                for (int i = 0; i < E * NW; i += 64) {
                    const uint32_t c = i + lane < E * NW ? tally[i + lane] : 0u;
                    const uint32_t s = wave_scan(c);
                    if (i + lane < E * NW)
                        tally[i + lane] = base + s - c;
                    base += (uint32_t)__shfl((int)s, 63, 64);
                }
            }
            __syncthreads();
        };
        uint64_t eqs[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int t = e * kPick + tid;
            eqs[e] = __ballot(want > 0 && t >= lo && t < hi && weight_key(x[e]) == key);
            if (lane == 0)
                tally[e * NW + wv] = (uint32_t)__popcll(eqs[e]);
        }
        scan();
        uint32_t keep = 0;
        uint32_t mine[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int t = e * kPick + tid;
            const bool middle = t >= lo && t < hi, eq = (eqs[e] >> lane) & 1;
            const uint32_t rank = tally[e * NW + wv] + (uint32_t)__popcll(eqs[e] & below);
            const bool k = t < len && (!middle || (want > 0 && (weight_key(x[e]) > key || (eq && rank < left))));
            keep |= (uint32_t)k << e;
            const uint64_t ks = __ballot(k);
            mine[e] = (uint32_t)__popcll(ks & below);
            eqs[e] = ks;
        }
        __syncthreads();
        if (lane == 0) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                tally[e * NW + wv] = (uint32_t)__popcll(eqs[e]);
        }
        scan();
#pragma unroll
        for (int e = 0; e < E; ++e)
            if ((keep >> e) & 1)
                put(e * kPick + tid, x[e], tally[e * NW + wv] + mine[e]);
    } else {
        __shared__ uint32_t wcount[2][NW];
        uint32_t base = 0, equal = 0;
        for (int t0 = 0; t0 < len; t0 += kPick) {
            const int t = t0 + tid;
            const bool in = t < len, middle = in && t >= lo && t < hi;
            const float xt = in ? w[t] : 0.f;
            const uint32_t k = weight_key(xt);
            const bool eq = middle && want > 0 && k == key;
            const uint64_t eqs = __ballot(eq);
            if (lane == 0)
                wcount[0][wv] = (uint32_t)__popcll(eqs);
            __syncthreads();
            uint32_t rank = equal + (uint32_t)__popcll(eqs & below);
            for (int i = 0; i < NW; ++i) {
                const uint32_t c = wcount[0][i];
                rank += i < wv ? c : 0u;
                equal += c;
            }
            const bool keep = in && (!middle || (want > 0 && (k > key || (eq && rank < left))));
            const uint64_t ks = __ballot(keep);
            if (lane == 0)
                wcount[1][wv] = (uint32_t)__popcll(ks);
            __syncthreads();
            uint32_t at = base + (uint32_t)__popcll(ks & below);
            for (int i = 0; i < NW; ++i) {
                const uint32_t c = wcount[1][i];
                at += i < wv ? c : 0u;
                base += c;
            }
            if (keep)
                put(t, xt, at);
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
    // (all rows' loads of a step at once: the chain is paid once, not per row)
    i32x4 code[NP];
    int ex[NP], from[NP], tok[NP];
    int e = -127;       // the block's exponent (of codes and bytes: the values may lie past FP32's largest)
#pragma unroll
    for (int q = 0; q < NP; ++q)
        tok[q] = kept[min(q * TPP + tk, z - 1)];
#pragma unroll
    for (int q = 0; q < NP; ++q)
        from[q] = page_of(p.bt, p.from.n_pages, b, max(tok[q], 0) / PAGE);
#pragma unroll
    for (int q = 0; q < NP; ++q) {
        const size_t at = (size_t)max(from[q], 0) * p.from.Hkv + hk;
        code[q] = *reinterpret_cast<const i32x4*>(src + at * (PAGE * D) + (max(tok[q], 0) % PAGE) * D + 16 * u);
        ex[q] = (int)src_scale[at] - 127;
    }
#pragma unroll
    for (int q = 0; q < NP; ++q) {
        if (from[q] < 0) {                          // (no page: zeros)
            code[q] = i32x4{};
            ex[q] = 0;
        }
        float top = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float y[4];
            from_e4m3((uint32_t)code[q][c], y);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top = fmax_f(top, __builtin_fabsf(y[e]));   // (a NaN code does not count)
        }
        if (q * TPP + tk < z && top > 0.f)
            e = max(e, block_exponent(top) + ex[q]);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        e = max(e, __shfl_xor(e, off, 64));
    __shared__ int wave_max[4];
    if ((threadIdx.x & 63) == 0)
        wave_max[threadIdx.x >> 6] = e;
    __syncthreads();
    e = max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3]));
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
    const int64_t heads = (int64_t)p.bt.B * p.from.Hkv;
    unsigned picks, moves;
    hipError_t e = grid_of(heads, kPick, picks);
    if (e == hipSuccess)
        e = grid_of((__int128)heads * p.nb * 2, 256, moves);
    if (e != hipSuccess)
        return e;
    const int most = p.bt.W * page;
    auto pick = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(picks), dim3(kPick), 0, s, p, most); };
    if (most <= 4 * kPick)
        pick(evict_pick<4>);
    else if (most <= 8 * kPick)
        pick(evict_pick<8>);
    else if (most <= 16 * kPick)
        pick(evict_pick<16>);
    else
        pick(evict_pick<0>);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(moves), dim3(256), 0, s, p);
        return hipGetLastError();
    };
    if (d == 64)
        return page == 64 ? go(evict_move<64, 64>) : go(evict_move<64, 128>);
    return page == 64 ? go(evict_move<128, 64>) : go(evict_move<128, 128>);
}

}  // namespace attn
