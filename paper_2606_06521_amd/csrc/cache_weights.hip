// Attention weight that cached tokens receive: per key the sum over the query
// rows of exp2(x - lse).
//
// D = Q K^T on the bf16 MFMA with the keys as columns: lane (n, g) holds rows
// 4 g .. 4 g + 3 of a 16-row tile for key n, so the sum over rows stays in the
// lane until the last row, and a key is owned by one wave: no atomics, one order
// of sums.  A wave takes the 128 keys of a visit; their codes lie in its LDS
// stage, widened to bf16 registers once for all row tiles.  With few rows it is
// bound by the stream of K, with many by the exp2 of every (row, key).
#include "cache_common.hpp"

#include <type_traits>

namespace attn {

namespace {

__device__ inline bf16x8 widen_w(uint32_t a, uint32_t b)
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const bf2 x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return bf16x8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}

template <int D, int PAGE, bool E4M3>
__global__ void __launch_bounds__(256) cache_weights_kernel(WeightParams p, int visits)
{
    constexpr int NW = 4;
    constexpr int KT = kVisit / 16, KP = D / 64;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int n = lane & 15, g = lane >> 4;
    const int groups = (visits + NW - 1) / NW;
    const int v = (int)(blockIdx.x % groups) * NW + w;
    const int rest = (int)(blockIdx.x / groups);
    const int hk = rest % p.cache.Hkv, b = rest / p.cache.Hkv;
    const Seq s = sequence(p.bt, b, p.max_len);
    const int t0 = v * kVisit;
    if (t0 >= s.len || s.n <= 0)
        return;

    // K operand: key 16 kt + n, channels 64 i + 16 g on (two k-steps)
    bf16x8 kf[KT][2 * KP];
    float c[KT], sum[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const int t = t0 + 16 * kt + n;
        const int pid = t < s.len ? page_of(p.bt, p.cache.n_pages, b, t / PAGE) : -1;
        const size_t block = (size_t)(pid < 0 ? 0 : pid) * p.cache.Hkv + hk;
        const uint8_t* row = p.cache.k + block * (PAGE * D) + (t % PAGE) * D;
        // (no key: a scale of NaN marks it)
        c[kt] = pid < 0 ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(p.c, (int)p.cache.ks[block] - 127);
        sum[kt] = 0.f;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const i32x4 x = pid < 0 ? i32x4{} : *reinterpret_cast<const i32x4*>(row + 64 * i + 16 * g);
            kf[kt][2 * i] = widen_w((uint32_t)x[0], (uint32_t)x[1]);
            kf[kt][2 * i + 1] = widen_w((uint32_t)x[2], (uint32_t)x[3]);
        }
    }

    const int rows = s.n * p.G;
    // (causal: the rows before the first that sees key t0 add nothing)
    const int first = p.causal ? max(t0 - s.pos0, 0) * p.G / 16 : 0;
    for (int tile = first; 16 * tile < rows; ++tile) {
        const int row = 16 * tile + n;
        bf16x8 qf[2 * KP];
        {
            const int i = row / p.G;
            const int64_t at = (int64_t)(s.first + i) * p.q.st + (int64_t)(hk * p.G + (row - i * p.G)) * p.q.sh;
#pragma unroll
            for (int j = 0; j < 2 * KP; ++j) {
                const int64_t e = at + 64 * (j / 2) + 16 * g + 8 * (j % 2);
                if (row >= rows) {
                    qf[j] = bf16x8{};
                } else if constexpr (E4M3) {
                    const i32x2 x = *reinterpret_cast<const i32x2*>(static_cast<const uint8_t*>(p.q.data) + e);
                    qf[j] = widen_w((uint32_t)x[0], (uint32_t)x[1]);
                } else {
                    qf[j] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const i32x4*>(static_cast<const uint16_t*>(p.q.data) + e));
                }
            }
        }
        // of the lane's four rows: lse in units of log2 (none: +inf, whose weights are 0), last key seen
        float lse2[4];
        int last[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int R = 16 * tile + 4 * g + r, i = R / p.G;
            lse2[r] = INFINITY;
            last[r] = -1;
            if (R < rows) {
                const float x = p.lse[(int64_t)(s.first + i) * p.Hq + hk * p.G + (R - i * p.G)];
                lse2[r] = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
                last[r] = p.causal ? s.pos0 + i : s.len - 1;
            }
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            f32x4 acc = {};
#pragma unroll
            for (int j = 0; j < 2 * KP; ++j)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[j], kf[kt][j], acc, 0, 0, 0);
            const int t = t0 + 16 * kt + n;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[r], c[kt], -lse2[r]));
                sum[kt] += t <= last[r] ? x : 0.f;
            }
        }
    }
    float* const out = p.w + (int64_t)b * p.sb + (int64_t)hk * p.sh;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        float x = sum[kt];
        x += __shfl_xor(x, 16, 64);
        x += __shfl_xor(x, 32, 64);
        const int t = t0 + 16 * kt + n;
        // (c = NaN: no page)
        if (g == 0 && t < s.len && c[kt] == c[kt])
            out[t] += x;
    }
}

}  // namespace

hipError_t launch_cache_weights(const WeightParams& p, int d, int page, bool e4m3, hipStream_t s)
{
    const int visits = (p.max_len + kVisit - 1) / kVisit;
    const int64_t grid = (int64_t)((visits + 3) / 4) * p.bt.B * p.cache.Hkv;
    if (grid > 1 << 30)
        return hipErrorInvalidValue;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, s, p, visits);
        return hipGetLastError();
    };
    auto by_type = [&](auto dc, auto pc) {
        constexpr int D = decltype(dc)::value, PAGE = decltype(pc)::value;
        return e4m3 ? go(cache_weights_kernel<D, PAGE, true>) : go(cache_weights_kernel<D, PAGE, false>);
    };
    using std::integral_constant;
    if (d == 64)
        return page == 64 ? by_type(integral_constant<int, 64>{}, integral_constant<int, 64>{})
                          : by_type(integral_constant<int, 64>{}, integral_constant<int, 128>{});
    return page == 64 ? by_type(integral_constant<int, 128>{}, integral_constant<int, 64>{})
                      : by_type(integral_constant<int, 128>{}, integral_constant<int, 128>{});
}

}  // namespace attn
