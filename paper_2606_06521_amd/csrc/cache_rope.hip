// Rotary positions, and the write of new tokens into the cache.
//
// Both move 16 channels of a token per thread: the two runs of eight that the
// rotation pairs (i and i + rot / 2), or 16 in a row (interleaved pairs, and
// channels that are not rotated).  What bounds them is memory where there are
// many tokens (the heads of 8192 tokens x 32 x 128 in 28 us, 4.8 TB/s, the rate of a large
// copy; 8 KV heads appended along 39 us, 4.0 TB/s, of which 7 are the rotation in 64 bits),
// the chain of loads (length, page, scale, row) where there are few: 3.0 and 4.7 us.
#include "cache_common.hpp"

namespace attn {

namespace {

// The unit u of 16 channels: where its two runs of eight start.
__device__ inline void unit_at(const Rotation& r, bool rotates, int u, int& o1, int& o2)
{
    const bool half = rotates && r.layout == 0;
    o1 = half ? 8 * u : 16 * u;
    o2 = half ? 8 * u + r.rot / 2 : 16 * u + 8;
}

// cos and sin of the unit's eight pairs (a position outside the table: NaN).
__device__ inline void unit_table(const Rotation& r, int pos, int u, float* cs)
{
    const bool in = (uint32_t)pos < (uint32_t)r.n_pos;
    const f32x4* t = reinterpret_cast<const f32x4*>(r.table + (int64_t)(in ? pos : 0) * r.rot + 16 * u);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x4 v = t[j];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            cs[4 * j + e] = in ? v[e] : __builtin_nanf("");
    }
}

// x: 16 channels in the order of the unit's runs; rotates them in FP32.
__device__ inline void rotate32(const Rotation& r, float* x, const float* cs)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float& a = r.layout == 0 ? x[j] : x[2 * j];
        float& b = r.layout == 0 ? x[8 + j] : x[2 * j + 1];
        const float c = cs[2 * j], s = cs[2 * j + 1];
        const float p = __builtin_fmaf(a, c, -(b * s)), q = __builtin_fmaf(b, c, a * s);
        a = p;
        b = q;
    }
}

// A 64-bit value as FP32 with the last bit set where it is not exact: every later
// rounding to fewer bits is that of the 64-bit value (of at least 2^-126; smaller
// ones round to FP32's subnormals first).
__device__ inline float to_odd(double x)
{
    uint64_t u = __builtin_bit_cast(uint64_t, x);
    uint32_t lo = (uint32_t)u;
    lo = (lo & 0xE0000000u) | (lo & 0x1FFFFFFFu ? 0x20000000u : 0u);
    u = (u & 0xFFFFFFFF00000000ull) | lo;
    return (float)__builtin_bit_cast(double, u);
}

__device__ inline void rotate64(const Rotation& r, float* x, const float* cs)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float& a = r.layout == 0 ? x[j] : x[2 * j];
        float& b = r.layout == 0 ? x[8 + j] : x[2 * j + 1];
        const double c = cs[2 * j], s = cs[2 * j + 1];
        const double p = __builtin_fma((double)a, c, -((double)b * s)), q = __builtin_fma((double)b, c, (double)a * s);
        a = to_odd(p);
        b = to_odd(q);
    }
}

// 16 channels of token t, head h, at position pos
template <int TYPE>
__device__ inline void rope_unit(const Heads& x, const Heads& out, const Rotation& r, int64_t t, int h, int u, int pos)
{
    const bool rotates = 16 * u < r.rot;
    int o1, o2;
    unit_at(r, rotates, u, o1, o2);
    float v[16];
    const int64_t at = t * x.st + h * x.sh, to = t * out.st + h * out.sh;
    load8<TYPE>(x.data, at + o1, v);
    load8<TYPE>(x.data, at + o2, v + 8);
    if (rotates) {
        float cs[16];
        unit_table(r, pos, u, cs);
        rotate32(r, v, cs);
    }
    store8<TYPE>(out.data, to + o1, v);
    store8<TYPE>(out.data, to + o2, v + 8);
}

template <int TYPE>
__global__ void __launch_bounds__(256) rope_kernel(Heads x, Heads out, int64_t n, int H, int upt, Rotation r)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n)
        return;
    const int u = (int)(i % upt);
    const int64_t th = i / upt, t = th / H;
    rope_unit<TYPE>(x, out, r, t, (int)(th - t * H), u, r.positions[t]);
}

// One workgroup per block that gets tokens, KV head, and K or V; behind them
// workgroups that rotate q.  The block's new values stay in registers between
// the pass that takes their largest and the one that writes their codes.
template <int TYPE, int D, int PAGE>
__global__ void __launch_bounds__(256) append_kernel(Batch bt, Cache cache, Heads k, Heads v, Rotation r, Heads q, Heads q_out,
                                                     int Hq, int most, int64_t n_blocks, int64_t q_groups)
{
    constexpr int UPT = D / 16;                     // units per token
    constexpr int TPP = 256 / UPT;                  // tokens per pass
    constexpr int NP = PAGE / TPP < 1 ? 1 : PAGE / TPP;
    if (blockIdx.x >= n_blocks) {
        const int64_t g = (int64_t)blockIdx.x - n_blocks;
        const int b = (int)(g / q_groups);
        const int64_t i = (g - b * q_groups) * 256 + threadIdx.x, th = i / UPT, t = th / Hq;
        const Seq s = sequence(bt, b, bt.W * PAGE);
        if (t < s.n)
            rope_unit<TYPE>(q, q_out, r, s.first + t, (int)(th - t * Hq), (int)(i % UPT),
                            r.positions ? r.positions[s.first + t] : s.pos0 + (int)t);
        return;
    }
    int64_t i = blockIdx.x;
    const bool is_v = i & 1;
    i >>= 1;
    const int h = (int)(i % cache.Hkv);
    i /= cache.Hkv;
    const int j = (int)(i % most), b = (int)(i / most);
    const Seq s = sequence(bt, b, bt.W * PAGE);
    const int lo = max(s.pos0, 0), end = min(s.pos0 + s.n, s.len);   // tokens [lo, end) are written
    if (end <= lo)
        return;
    const int block = lo / PAGE + j;
    const int t0 = block * PAGE;
    if (t0 >= end)
        return;
    const int pid = page_of(bt, cache.n_pages, b, block);
    if (pid < 0)
        return;
    const int a = max(lo - t0, 0), z = min(end - t0, PAGE);   // slots [a, z) are new, [0, a) older
    uint8_t* const codes = (is_v ? cache.v : cache.k) + ((size_t)pid * cache.Hkv + h) * (PAGE * D);
    uint8_t* const scale = (is_v ? cache.vs : cache.ks) + (size_t)pid * cache.Hkv + h;
    const Heads& x = is_v ? v : k;

    const int u = threadIdx.x % UPT, tk = threadIdx.x / UPT;
    const bool rotates = !is_v && r.table && 16 * u < r.rot;
    int o1, o2;
    unit_at(r, rotates, u, o1, o2);
    // (all loads of a step at once: the chain is paid once, not per token; slots past
    // the last new one read that one again)
    float val[NP][16];
    int pos[NP];
    const int was = a > 0 ? (int)*scale - 127 : -128;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        if (p * TPP >= z - a)
            break;
        const int slot = min(a + p * TPP + tk, z - 1);
        const int t = t0 + slot - s.pos0 + s.first;     // the packed token
        const int64_t at = (int64_t)t * x.st + (int64_t)h * x.sh;
        pos[p] = rotates && r.positions ? r.positions[t] : t0 + slot;
        load8<TYPE>(x.data, at + o1, val[p]);
        load8<TYPE>(x.data, at + o2, val[p] + 8);
    }
    if (rotates) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (p * TPP >= z - a)
                break;
            float cs[16];
            unit_table(r, pos[p], u, cs);
            rotate64(r, val[p], cs);
        }
    }
    float amax = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        if (p * TPP >= z - a)
            break;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float m = __builtin_fabsf(val[p][e]);
            const bool finite = m < __builtin_inff();
            amax = fmax_f(amax, finite ? m : 0.f);
            val[p][e] = finite ? val[p][e] : __builtin_nanf("");
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        amax = fmax_f(amax, __shfl_xor(amax, off, 64));
    __shared__ float wave_max[4];
    if ((threadIdx.x & 63) == 0)
        wave_max[threadIdx.x >> 6] = amax;
    __syncthreads();
    amax = fmax_f(fmax_f(wave_max[0], wave_max[1]), fmax_f(wave_max[2], wave_max[3]));
    const int e = max(block_exponent(amax), was);
    if (threadIdx.x == 0)
        *scale = (uint8_t)(e + 127);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int slot = a + p * TPP + tk;
        if (slot >= z)
            continue;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float y[8];
#pragma unroll
            for (int m = 0; m < 8; ++m)
                y[m] = __builtin_amdgcn_ldexpf(val[p][8 * c + m], -e);
            *reinterpret_cast<i32x2*>(codes + slot * D + (c ? o2 : o1)) =
                i32x2{(int)to_e4m3(y[0], y[1], y[2], y[3]), (int)to_e4m3(y[4], y[5], y[6], y[7])};
        }
    }
    // older codes on the grown scale
    if (a > 0 && e > was) {
        for (int i = threadIdx.x; i < a * D / 16; i += 256) {
            i32x4 w = *reinterpret_cast<const i32x4*>(codes + 16 * i);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float y[4];
                from_e4m3((uint32_t)w[c], y);
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    y[m] = __builtin_amdgcn_ldexpf(y[m], was - e);
                w[c] = (int)to_e4m3(y[0], y[1], y[2], y[3]);
            }
            *reinterpret_cast<i32x4*>(codes + 16 * i) = w;
        }
    }
}

}  // namespace

hipError_t launch_rope(const Heads& x, const Heads& out, int T, int H, int d, int type, const Rotation& r, hipStream_t s)
{
    const int upt = d / 16;
    unsigned grid;
    const __int128 units = (__int128)T * H * upt;
    const hipError_t e = grid_of((units + 255) / 256, 256, grid);
    if (e != hipSuccess)
        return e;
    const int64_t n = (int64_t)units;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, x, out, n, H, upt, r);
        return hipGetLastError();
    };
    return type == kTypeF32 ? go(rope_kernel<kTypeF32>) : type == kTypeBf16 ? go(rope_kernel<kTypeBf16>) : go(rope_kernel<kTypeF16>);
}

hipError_t launch_append(const Batch& bt, const Cache& c, int d, int page, const Heads& k, const Heads& v, int type,
                         const Rotation& r, const Heads& q, const Heads& q_out, int Hq, hipStream_t s)
{
    // blocks that max_q tokens can lie in
    const int most = (int)(((int64_t)bt.max_q + page - 2) / page + 1);
    const __int128 writes = (__int128)bt.B * most * c.Hkv * 2;
    const int64_t q_groups = q.data ? ((int64_t)bt.max_q * Hq * (d / 16) + 255) / 256 : 0;   // of a sequence
    unsigned grid;
    const hipError_t e = grid_of(writes + (__int128)bt.B * q_groups, 256, grid);
    if (e != hipSuccess)
        return e;
    const int64_t blocks = (int64_t)writes;
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, bt, c, k, v, r, q, q_out, Hq, most, blocks, q_groups);
        return hipGetLastError();
    };
    auto by_type = [&](auto ty) {
        constexpr int TY = decltype(ty)::value;
        if (d == 64)
            return page == 64 ? go(append_kernel<TY, 64, 64>) : go(append_kernel<TY, 64, 128>);
        return page == 64 ? go(append_kernel<TY, 128, 64>) : go(append_kernel<TY, 128, 128>);
    };
    using std::integral_constant;
    return type == kTypeF32    ? by_type(integral_constant<int, kTypeF32>{})
           : type == kTypeBf16 ? by_type(integral_constant<int, kTypeBf16>{})
                               : by_type(integral_constant<int, kTypeF16>{});
}

}  // namespace attn
