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
// which 32 rows share: 74 % of the cycles, beside 42 % of the matrix cores' (counted in a
// run of 448 us).  8 heads x 2048 x 4 rows against 16384 keys, d = 128: 408 us, 1.26 PFLOP/s
// (2 % more or less from card to card); a large bf16 product reaches 1.40.
#pragma once

#include "cache_fwd_kernel.hpp"

namespace attn {

constexpr int kTileRows = 128;
constexpr int kTileChunk = 512;     // visits of a range

template <int D, int PAGE, bool E4M3, class P>
__global__ void __launch_bounds__(256, 2) cache_fwd_tile_kernel(P p)
{
    constexpr int NW = 4, TR = kTileRows;
    constexpr int PPV = kVisit / PAGE;          // pages per visit
    constexpr int DT = D / 32;                  // d tiles of O^T
    constexpr int KT = kVisit / 32;             // S^T tiles per visit
    constexpr int KP = D / 32;                  // 16-byte pieces of a key row per lane (two k-steps each)
    constexpr int CPR = D / 16;                 // 16-byte chunks per row
    constexpr int STAGE = kVisit * D;           // bytes of a K or V stage
    constexpr int LPW = STAGE / 1024 / NW;      // loads per stage and wave
    constexpr int RPI = 1024 / D;               // rows per load
    static_assert(LPW * RPI == 32, "a wave loads 32 rows, of one page");

    __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * STAGE];     // K, V, K, V
    __shared__ int pids[kTileChunk * PPV];
    __shared__ uint8_t kbyte[kTileChunk * PPV], vbyte[kTileChunk * PPV];

    __shared__ int starts[kLists<P> ? kTileChunk * PPV : 1];     // first keys of a list's pages
    __shared__ int row_last[kShared<P> ? TR : 1];

    Share x;
    if (!share_of(p, TR, PAGE, x))
        return;
    const Seq& s = x.u.s;
    const int rows = s.n * p.gr.G, row0 = x.tile * TR, hk = x.u.hk;
    const int v0 = x.v0;
    int v1 = x.v1;

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, h = lane >> 5;
    const int wrow0 = row0 + 32 * w;                    // the wave's first row
    const int row = wrow0 + n;
    int pos = row < rows ? last_key(s.pos0 + p.gr.token(row), p.causal, s.len) : -1;
    int pos_min = last_key(s.pos0 + p.gr.token(wrow0), p.causal, s.len);
    int tile_pos_min = last_key(s.pos0 + p.gr.token(row0), p.causal, s.len), seen = tile_seen(p, s, x.tile, TR);
    if constexpr (kShared<P>)
        if (x.u.common) {
            common_last(p, row0, TR, row_last);
            pos = row_last[32 * w + n];
            int lo = pos, all = min(row_last[lane], row_last[lane + 64]), hi = max(row_last[lane], row_last[lane + 64]);
#pragma unroll
            for (int off = 16; off > 0; off >>= 1)
                lo = min(lo, __shfl_xor(lo, off, 64));
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) {
                all = min(all, __shfl_xor(all, off, 64));
                hi = max(hi, __shfl_xor(hi, off, 64));
            }
            pos_min = __builtin_amdgcn_readfirstlane(lo);
            tile_pos_min = __builtin_amdgcn_readfirstlane(all);
            seen = min(p.shared * PAGE, min(__builtin_amdgcn_readfirstlane(hi), p.max_len - 1) + 1);
        }

    const int np = max(v1 - v0, 0) * PPV;
    for (int i = tid; i < np; i += 256) {
        const int at = v0 * PPV + i;
        if constexpr (kLists<P>) {
            const int block = at < p.take ? x.u.list[at] : -1;
            pids[i] = page_of(p.bt, p.cache.n_pages, x.u.b, block);
            starts[i] = pids[i] < 0 ? 0 : block * PAGE;
        } else {
            pids[i] = x.u.common && at >= shared_pages(p) ? -1 : page_of(p.bt, p.cache.n_pages, x.u.b, x.u.base + at);
        }
    }
    __syncthreads();
    if constexpr (kLists<P>)
        v1 = listed_end<PPV>(pids, v0, np, lane);
    // first key of the range's page i
    auto start = [&](int i) __attribute__((always_inline)) {
        if constexpr (kLists<P>)
            return i < np ? starts[i] : 0;
        else
            return (x.u.base + v0 * PPV + i) * PAGE;
    };

    const size_t block_bytes = (size_t)PAGE * D;
    const int lr = lane / CPR, lc = lane % CPR;
    auto vswz = [](int r) __attribute__((always_inline)) { return ((r / (256 / D)) & (CPR / 2 - 1)) * 2; };
    auto kswz = [](int r) __attribute__((always_inline)) {
        return D == 128 ? ((r & 3) | ((r >> 4) & 1) << 2) : (((r >> 1) & 1) | ((r >> 4) & 1) << 1);
    };
    const int k_off = lr * D + 16 * (lc ^ (D == 128 ? (lr & 3) : ((lr >> 1) & 1)));
    const int v_off = lr * D + 16 * (lc ^ vswz(lr));
    // the wave's rows 32 w .. 32 w + 31 of the visit's K and V, into stage pair v & 1
    auto issue = [&](int v) __attribute__((always_inline)) {
        const int sub = PPV == 2 ? w >> 1 : 0;
        const int i = (v - v0) * PPV + sub;
        const int pid = v < v1 ? __builtin_amdgcn_readfirstlane(pids[i]) : -1;
        const int from = kLists<P> ? __builtin_amdgcn_readfirstlane(start(i)) : start(i);
        const int left = pid < 0 ? 0 : min(max(seen - from, 0), PAGE) * D;
        const size_t at = ((size_t)(pid < 0 ? 0 : pid) * p.cache.Hkv + hk) * block_bytes;
        const i32x4 kb = bytes_buffer(p.cache.k + at, left), vb = bytes_buffer(p.cache.v + at, left);
        const uint8_t* const st = lds + (v & 1) * 2 * STAGE + w * (32 * D);
        const int src = (32 * w - sub * PAGE) * D;
#pragma unroll
        for (int j = 0; j < LPW; ++j)
            load_lds16(kb, k_off ^ (((RPI * j) >> 4) & 1 ? (D == 128 ? 64 : 32) : 0), src + 1024 * j, st + 1024 * j);
#pragma unroll
        for (int j = 0; j < LPW; ++j)
            load_lds16(vb, v_off, src + 1024 * j, st + STAGE + 1024 * j);
    };
    // the first visit's K and V travel while the scales and Q arrive
    issue(v0);
    for (int i = tid; i < np; i += 256) {
        // (a page behind the last key that a row sees may hold anything)
        const int pid = start(i) < seen ? pids[i] : -1;
        const size_t at = (size_t)(pid < 0 ? 0 : pid) * p.cache.Hkv + hk;
        kbyte[i] = pid < 0 ? 127 : p.cache.ks[at];
        vbyte[i] = pid < 0 ? 127 : p.cache.vs[at];
    }
    bf16x8 qf[2 * KP];
    {
        // (rows past the last take its Q and are not written)
        const int at_row = min(row, rows - 1), i = p.gr.token(at_row);
        const int64_t at = (int64_t)(s.first + i) * p.q.st + (int64_t)(hk * p.gr.G + (at_row - i * p.gr.G)) * p.q.sh;
#pragma unroll
        for (int j = 0; j < 2 * KP; ++j)
            qf[j] = load_q8<E4M3>(p.q.data, at + 32 * (j / 2) + 16 * h + 8 * (j % 2));
    }

    // (of the wave's rows, in a scalar register; NaN of a row does not count)
    float far = far_factor<2 * KP>(qf, D);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        far = fmax_f(far, __shfl_xor(far, off, 64));
    far = __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(far)));
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
        o[dt] = f32x16{};
    float ell = 0.f, ref = -INFINITY;

    const int krow = a_row_to_key(n);
    const int j16 = lane & 15;
    const uint32_t v_lane = (uint32_t)(((j16 >> 1) + 16 * h) * D + (((n >> 4) ^ vswz(j16 >> 1)) << 4) + 8 * (j16 & 1));

    for (int v = v0; v < v1; ++v) {
        // this visit's K and V are there, and everyone is done with the other pair
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        issue(v + 1);
        uint8_t* const kst = lds + (v & 1) * 2 * STAGE;
        uint8_t* const vst = kst + STAGE;
        const int pi = (v - v0) * PPV;
        const int t0[2] = {start(pi), PPV == 2 ? start(pi + 1) : start(pi) + 64};    // of its halves
        const int t_end = kLists<P> ? max(t0[0], t0[1]) + 64 : t0[1] + 64;
        auto v_read = [&](int js, int dt) __attribute__((always_inline)) {
            i32x8 av;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const i32x2 t = read_tr8(vst + (v_lane ^ (uint32_t)(dt << 5)) + (64 * js + 32 * (u / 2) + 8 * (u % 2)) * D);
                av[2 * u] = t[0];
                av[2 * u + 1] = t[1];
            }
            return av;
        };
        // Where some rows see keys that others do not, a NaN of V must not reach the others
        // by way of 0 times NaN: it makes NaN of the sums of the rows that see it, and goes
        // (every wave looks at the whole stage, so all take the same way).
        if (t_end - 1 > tile_pos_min && holds_nan(vst, STAGE, lane)) {
#pragma unroll
            for (int js = 0; js < KT / 2; ++js) {
                i32x8 see;
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    see[q] = ones(pos - t0[js] - 32 * (q / 4) - 16 * h - 4 * (q % 4) + 1);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const f32x16 hits = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(nan_ones(v_read(js, dt)), see, f32x16{}, 0, 0, 0, 127, 0, 127);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        o[dt][r] = hits[r] > 0.f ? __builtin_nanf("") : o[dt][r];
                }
            }
            lds_barrier();
            clear_nans(vst + w * (32 * D), 32 * D, lane);
            lds_barrier();
        }
        if (wrow0 >= rows)
            continue;
        float c[2] = {score_factor(p.c, kbyte[pi]), score_factor(p.c, kbyte[pi + PPV - 1])};
        const int lent[2] = {lent_scale(vbyte[pi]), lent_scale(vbyte[pi + PPV - 1])};
        const int sa[2] = {vbyte[pi] - lent[0], vbyte[pi + PPV - 1] - lent[1]};
        const bool there[2] = {pids[pi] >= 0, pids[pi + PPV - 1] >= 0};
        f32x16 sc[KT];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const int r = krow + 32 * kt;
            f32x16 acc = {};
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const i32x4 k = *reinterpret_cast<const i32x4*>(kst + r * D + 16 * ((2 * i + h) ^ kswz(r)));
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((uint32_t)k[0], (uint32_t)k[1]), qf[2 * i], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen((uint32_t)k[2], (uint32_t)k[3]), qf[2 * i + 1], acc, 0, 0, 0);
            }
            sc[kt] = acc;
        }
        __builtin_amdgcn_s_setprio(0);
        // ---- keys the row does not see ----
        if (t_end - 1 > pos_min || !there[0] || !there[1]) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int lim = there[kt / 2] ? pos - t0[kt / 2] - 32 * (kt % 2) - 16 * h : -1;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sc[kt][r] = r <= lim ? sc[kt][r] : -INFINITY;
            }
        }
        // ---- P in units of 2^M, the least power of two not below the group's largest ----
        float M[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            float mx = sc[kt][0];
#pragma unroll
            for (int r = 1; r < 16; ++r)
                mx = max_of(mx, sc[kt][r]);
            mx = halves_max(mx);
            M[kt] = mx != mx ? 0.f : __builtin_ceilf(mx * c[kt / 2]);
        }
        // (there the FP32 products themselves are the scores)
        if (__ballot(fmax_f(c[0], c[1]) * far > 1.f) != 0) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sc[kt][r] *= c[kt / 2];
            c[0] = c[1] = 1.f;
        }
        const float hi = fmax_f(fmax_f(M[0], M[1]), fmax_f(M[2], M[3]));
        if (__ballot(hi > ref + kSlack) != 0) {
            const float to = hi > ref + kSlack ? hi : ref;
            const int down = shift_of(ref, to);
            ref = to;
            ell = __builtin_amdgcn_ldexpf(ell, down);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    o[dt][r] = __builtin_amdgcn_ldexpf(o[dt][r], down);
        }
        int pk[4 * KT], sb[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const bool none = M[kt] == -INFINITY;
            const float nm = none ? 0.f : -M[kt];
            const int up = (int)__builtin_fmaxf(none ? -300.f : M[kt] - ref, -300.f);
            float sum = 0.f;
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                float e[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][4 * r4 + r], c[kt / 2], nm));
                    sum += e[r];
                }
                s16x2 word = {};
                word = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(word, e[0], e[1], 0x1p-8f, false);
                word = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(word, e[2], e[3], 0x1p-8f, true);
                pk[4 * kt + r4] = __builtin_bit_cast(int, word);
            }
            ell += __builtin_amdgcn_ldexpf(sum, up);
            sb[kt] = max(127 - 8 + lent[kt / 2] + up, 0);
        }
        // ---- O^T += V^T P^T ----
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int js = 0; js < KT / 2; ++js) {
            // the first group's scale from the lower half, the second's from the upper
            const int scale_b = h ? sb[2 * js + 1] : sb[2 * js];
            i32x8 bop;
#pragma unroll
            for (int q = 0; q < 8; ++q)
                bop[q] = pk[8 * js + q];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const i32x8 av = v_read(js, dt);
                o[dt] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bop, o[dt], 0, 0, 0, sa[js], 0, scale_b);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (row >= rows)
        return;
    const float l = halves_sum(ell);
    if (x.whole) {
        const float inv = 1.f / l;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                write_row<D>(p, s, hk, row, 8 * dt + 2 * r4 + h, f32x4{o[dt][4 * r4], o[dt][4 * r4 + 1], o[dt][4 * r4 + 2], o[dt][4 * r4 + 3]},
                             l, inv, ref);
        return;
    }
    float* const part = part_of(p, x, TR, D);
    const int rr = 32 * w + n;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
            *reinterpret_cast<f32x4*>(part + rr * D + 32 * dt + 8 * r4 + 4 * h) =
                f32x4{o[dt][4 * r4], o[dt][4 * r4 + 1], o[dt][4 * r4 + 2], o[dt][4 * r4 + 3]};
    if (h == 0) {
        part[TR * D + rr] = l;
        part[TR * (D + 1) + rr] = ref;
    }
}

}  // namespace attn
