// Attention over the cache: tiles of 16 query rows, one wave per visit of 128 keys.
//
// The query heads of a group read the same keys: the rows of a (sequence, KV
// head) are its new tokens times the group's heads, row R = token R / G, head
// R % G, in tiles of 16.  A workgroup of four waves takes a range of a tile's
// visits, wave w every fourth one.
//
// S^T = K Q^T on the bf16 MFMA: E4M3 codes are bf16 numbers, so the scores of the
// codes are those of FP32 (the FP8 MFMA would drop what lies 13 bits below a
// group's largest product).  The tiles' keys are chosen so that lane (n, g) holds
// the scores of row n and keys 16 g .. 16 g + 15 of either half of the visit: the
// E4M3 bytes of P are then the operand of P.V as they stand, and a group of 32
// keys with its own power of two is what one scale of that operand covers: the
// 16 keys of two neighbouring lane groups.  So a group's maximum M_g takes one
// exchange of lanes; 2^(x - M_g) is rounded to E4M3 and M_g - M goes to the matrix
// core as the operand's scale, V's page scale as the other operand's.  (The core adds
// products in eights and drops what lies 13 bits below their largest: 6e-5 of the
// result, where a code is rounded at 2^-4; bf16 products run at half its rate.)  No
// accumulator is rescaled as long as the row's reference M, taken at its first
// keys, holds within 2^kSlack.  So the waves need no barrier until they add up
// their (O, l), and the result does not depend on how the visits are shared out
// but for the order of FP32 sums.
//
// K and V go straight from memory into the wave's LDS stages by 1 KB loads; K's codes
// go on to registers at once, so the next visit's K is on its way all through this one, and
// V from the end of P.V on: two stages of 16 KB per wave (d = 128) keep up to 128 KB in flight
// per CU.  What bounds it is that stream: 16 x 8 heads x 8192 keys, 4 rows each, 50 us, 5.4
// TB/s (a large read reaches 6.0), and 5 for the merge.
#pragma once

#include "cache_common.hpp"

namespace attn {

constexpr int kMaxChunk = 128;      // visits of a range (its page numbers are kept in LDS)
constexpr float kSlack = 16.f;      // how far (log2) a group's maximum may exceed the row's reference

// Visits of a tile: those that hold a key that its last row sees.
__device__ inline int tile_visits(const FwdParams& p, const Seq& s, int tile, int tile_rows)
{
    const int last = min((tile + 1) * tile_rows, s.n * p.gr.G) - 1;       // last row
    const int seen = p.causal ? min(max(s.pos0 + p.gr.token(last) + 1, 0), s.len) : s.len;
    return (seen + kVisit - 1) / kVisit;
}

// Workgroup -> tile, range, KV head and sequence.  Tiles run fastest and each XCD
// takes a contiguous run: the tiles that read the same keys share an L2.
__device__ inline bool workgroup_of(const FwdParams& p, int& tile, int& range, int& hk, int& b)
{
    const int total = p.bt.B * p.cache.Hkv * p.ranges * p.tiles;
    const int per_xcd = (total + kNumXcd - 1) / kNumXcd;
    const int slot = (int)(blockIdx.x / kNumXcd), L = (int)(blockIdx.x % kNumXcd) * per_xcd + slot;
    if (slot >= per_xcd || L >= total)
        return false;
    tile = p.tiles - 1 - L % p.tiles;           // (causal: the longest first)
    int rest = L / p.tiles;
    range = rest % p.ranges;
    rest /= p.ranges;
    hk = rest % p.cache.Hkv;
    b = rest / p.cache.Hkv;
    return true;
}

// Four channels of a row's result: acc / l (inv = 1 / l), in units of 2^m.
template <int D>
__device__ inline void write_row(const FwdParams& p, const Seq& s, int hk, int R, int piece, f32x4 acc, float l, float inv, float m)
{
    const int i = p.gr.token(R);
    const int64_t row = (int64_t)(s.first + i) * p.Hq + hk * p.gr.G + (R - i * p.gr.G);
    // (no key seen: l = 0, m = -inf)
#pragma unroll
    for (int e = 0; e < 4; ++e)
        acc[e] = m == -INFINITY ? 0.f : acc[e] * inv;
    if (p.out_bf16) {
        const uint32_t lo = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)acc[0]) |
                            (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)acc[1]) << 16;
        const uint32_t hi = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)acc[2]) |
                            (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)acc[3]) << 16;
        *reinterpret_cast<i32x2*>(static_cast<uint16_t*>(p.out) + row * D + 4 * piece) = i32x2{(int)lo, (int)hi};
    } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + row * D + 4 * piece) = acc;
    }
    if (p.lse && piece == 0)
        p.lse[row] = m == -INFINITY ? -INFINITY : (m + __builtin_log2f(l)) * 0.6931471805599453f;
}

template <int D, int PAGE, bool E4M3>
__global__ void __launch_bounds__(256, 1) cache_fwd_kernel(FwdParams p)
{
    constexpr int NW = 4, TR = 16;
    constexpr int PPV = kVisit / PAGE;          // pages per visit
    constexpr int DT = D / 16;                  // d tiles of O^T
    constexpr int KT = kVisit / 16;             // S^T tiles per visit
    constexpr int KP = D / 64;                  // 16-byte pieces of a key row per lane (two k-steps each)
    constexpr int CPR = D / 16;                 // 16-byte chunks per row
    constexpr int STAGE = kVisit * D;           // bytes of a K or V stage
    constexpr int NI = STAGE / 1024;            // loads per stage
    constexpr int RPI = 1024 / D;               // rows per load
    constexpr int IPP = NI / PPV;               // loads per page
    constexpr int MS = D + 4;                   // row stride of the merge buffer (floats)
    static_assert(NW * TR * MS * 4 <= NW * 2 * STAGE, "the merge buffer takes the stages' place");

    __shared__ __attribute__((aligned(1024))) uint8_t lds[NW * 2 * STAGE];
    __shared__ int pids[kMaxChunk * PPV];
    __shared__ uint8_t kbyte[kMaxChunk * PPV], vbyte[kMaxChunk * PPV];
    __shared__ float lsh[NW][TR], msh[NW][TR];

    int tile, range, hk, b;
    if (!workgroup_of(p, tile, range, hk, b))
        return;
    const Seq s = uniform(sequence(p.bt, b, p.max_len));
    const int rows = s.n * p.gr.G;
    const int row0 = tile * TR;
    if (row0 >= rows)
        return;
    const int visits = tile_visits(p, s, tile, TR);
    const int v0 = range * p.chunk, v1 = min(v0 + p.chunk, visits);
    if (v0 >= v1 && range > 0)
        return;
    const bool whole = visits <= p.chunk;               // the only range of the tile

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int row = row0 + n;
    const int pos = row < rows ? last_key(s.pos0 + p.gr.token(row), p.causal, s.len) : -1;
    const int pos_min = last_key(s.pos0 + p.gr.token(row0), p.causal, s.len);
    const int seen = p.causal ? min(max(s.pos0 + p.gr.token(min(row0 + TR, rows) - 1) + 1, 0), s.len) : s.len;

    // the range's page numbers, then their scales
    const int np = max(v1 - v0, 0) * PPV;
    for (int i = tid; i < np; i += 256)
        pids[i] = page_of(p.bt, p.cache.n_pages, b, v0 * PPV + i);
    __syncthreads();

    const size_t block_bytes = (size_t)PAGE * D;
    uint8_t* const kst = lds + w * 2 * STAGE;
    uint8_t* const vst = kst + STAGE;
    // K stage: row r's chunk c at chunk c ^ kswz(r): the 16 rows of an operand read
    // (16 i + 4 kt + j, i and j < 4) fall in distinct banks eight at a time
    const int lr = lane / CPR, lc = lane % CPR;
    const int kswz_lane = D == 128 ? (lr & 3) : ((lr >> 1) & 1);
    const int k_off = lr * D + 16 * (lc ^ kswz_lane);
    // V stage: the layout ds_read_b64_tr_b8 takes without bank conflicts
    auto vswz = [](int r) __attribute__((always_inline)) { return ((r / (256 / D)) & (CPR / 2 - 1)) * 2; };
    const int v_off = lr * D + 16 * (lc ^ vswz(lr));
    // the part of page i (of the range) that the tile sees; no page: no bytes
    auto buffer = [&](const uint8_t* base, int v, int sub) __attribute__((always_inline)) {
        const int i = (v - v0) * PPV + sub;
        const int pid = v < v1 ? __builtin_amdgcn_readfirstlane(pids[i]) : -1;
        const int left = min(max(seen - (v * kVisit + sub * PAGE), 0), PAGE);
        return bytes_buffer(base + ((size_t)(pid < 0 ? 0 : pid) * p.cache.Hkv + hk) * block_bytes, pid < 0 ? 0 : left * D);
    };
    auto issue_k = [&](int v) __attribute__((always_inline)) {
#pragma unroll
        for (int sub = 0; sub < PPV; ++sub) {
            const auto kb = buffer(p.cache.k, v, sub);
#pragma unroll
            for (int j = 0; j < IPP; ++j) {
                const int i = sub * IPP + j;
                // bit 4 of the row (a row of the second, fourth 16) is the swizzle's next bit
                const int flip = ((RPI * i) >> 4) & 1 ? (D == 128 ? 64 : 32) : 0;
                load_lds16(kb, k_off ^ flip, 1024 * j, kst + 1024 * i);
            }
        }
    };
    auto issue_v = [&](int v) __attribute__((always_inline)) {
#pragma unroll
        for (int sub = 0; sub < PPV; ++sub) {
            const auto vb = buffer(p.cache.v, v, sub);
#pragma unroll
            for (int j = 0; j < IPP; ++j)
                load_lds16(vb, v_off, 1024 * j, vst + 1024 * (sub * IPP + j));
        }
    };

    // the first visit's K and V travel while the scales and Q arrive
    issue_k(v0 + w);
    issue_v(v0 + w);
    uint8_t kb0[(kMaxChunk * PPV + 255) / 256], vb0[(kMaxChunk * PPV + 255) / 256];
#pragma unroll
    for (int c = 0; c < (kMaxChunk * PPV + 255) / 256; ++c) {
        const int i = tid + 256 * c;
        // (a page behind the last key that a row sees may hold anything)
        const int pid = i < np && (v0 * PPV + i) * PAGE < seen ? pids[i] : -1;
        const size_t at = (size_t)(pid < 0 ? 0 : pid) * p.cache.Hkv + hk;
        kb0[c] = pid < 0 ? 127 : p.cache.ks[at];
        vb0[c] = pid < 0 ? 127 : p.cache.vs[at];
    }
    // Q^T fragments: k-step 2 i + e of lane (n, g): channels 64 i + 16 g + 8 e on
    bf16x8 qf[2 * KP];
    {
        // (rows past the last take its Q and are not written)
        const int at_row = min(row, rows - 1), i = p.gr.token(at_row);
        const int64_t at = (int64_t)(s.first + i) * p.q.st + (int64_t)(hk * p.gr.G + (at_row - i * p.gr.G)) * p.q.sh;
#pragma unroll
        for (int j = 0; j < 2 * KP; ++j)
            qf[j] = load_q8<E4M3>(p.q.data, at + 64 * (j / 2) + 16 * g + 8 * (j % 2));
    }
#pragma unroll
    for (int c = 0; c < (kMaxChunk * PPV + 255) / 256; ++c) {
        const int i = tid + 256 * c;
        if (i < np) {
            kbyte[i] = kb0[c];
            vbyte[i] = vb0[c];
        }
    }
    lds_barrier();

    const float far = far_factor<2 * KP>(qf, D);
    f32x4 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
        o[dt] = f32x4{};
    float ell = 0.f, ref = -INFINITY;       // l of the lane's keys and O of the row, in units of 2^ref

    // K operand of tile kt: rows 64 (kt / 4) + 16 (n >> 2) + 4 (kt % 4) + (n & 3), chunk 4 i + g
    const int krow = 16 * (n >> 2) + (n & 3);
    auto kswz = [](int r) __attribute__((always_inline)) {
        return D == 128 ? ((r & 3) | ((r >> 4) & 1) << 2) : (((r >> 1) & 1) | ((r >> 4) & 1) << 1);
    };
    // V^T operand: rows 64 (u / 2) + 16 g + 8 (u % 2) on, u < 4, chunk dt
    const int j16 = lane & 15;
    const uint32_t v_lane = (uint32_t)(((j16 >> 1) + 16 * g) * D + (vswz(j16 >> 1) << 4) + 8 * (j16 & 1));

    for (int v = v0 + w; v < v1; v += NW) {
        // the pages of the visit's two halves
        const int pi = (v - v0) * PPV;
        float c[2] = {score_factor(p.c, kbyte[pi]), score_factor(p.c, kbyte[pi + PPV - 1])};
        const int lent[2] = {lent_scale(vbyte[pi]), lent_scale(vbyte[pi + PPV - 1])};
        const int sa = vbyte[pi + (g >= 2 ? PPV - 1 : 0)] - (g >= 2 ? lent[1] : lent[0]);
        const bool there[2] = {pids[pi] >= 0, pids[pi + PPV - 1] >= 0};
        // ---- scores (K is older than V: wait for all but V's loads) ----
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NI) : "memory");
        i32x4 raw[KT][KP];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int r = krow + 64 * (kt / 4) + 4 * (kt % 4);
                raw[kt][i] = *reinterpret_cast<const i32x4*>(kst + r * D + 16 * ((4 * i + g) ^ kswz(r)));
            }
        // (all in registers: the stage takes the next visit)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        issue_k(v + NW);
        f32x4 sc[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            f32x4 acc = {};
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const i32x4 x = raw[kt][i];
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen((uint32_t)x[0], (uint32_t)x[1]), qf[2 * i], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen((uint32_t)x[2], (uint32_t)x[3]), qf[2 * i + 1], acc, 0, 0, 0);
            }
            sc[kt] = acc;
        }
        // ---- keys the row does not see ----
        const int t0 = v * kVisit;
        if (t0 + kVisit - 1 > pos_min || !there[0] || !there[1]) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int lim = there[kt / 4] ? pos - t0 - 64 * (kt / 4) - 16 * g : -1;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    sc[kt][r] = 4 * (kt % 4) + r <= lim ? sc[kt][r] : -INFINITY;
            }
        }
        // ---- P in units of 2^M, the least power of two not below the group's largest ----
        float M[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            float mx = sc[4 * hf][0];
#pragma unroll
            for (int i = 1; i < 16; ++i)
                mx = max_of(mx, sc[4 * hf + i / 4][i % 4]);
            const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmax_f(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
            // (all of them NaN: any M hands the NaN on)
            M[hf] = mx != mx ? 0.f : __builtin_ceilf(mx * c[hf]);
        }
        // (there the FP32 products themselves are the scores)
        if (__ballot(fmax_f(c[0], c[1]) * far > 1.f) != 0) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    sc[kt][r] *= c[kt / 4];
            c[0] = c[1] = 1.f;
        }
        const float hi = fmax_f(M[0], M[1]);
        if (__ballot(hi > ref + kSlack) != 0) {
            const float top = halves_max(hi);
            const float to = top > ref + kSlack ? top : ref;
            const int down = shift_of(ref, to);
            ref = to;
            ell = __builtin_amdgcn_ldexpf(ell, down);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    o[dt][r] = __builtin_amdgcn_ldexpf(o[dt][r], down);
        }
        i32x8 pk;
        uint32_t sb[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const bool none = M[hf] == -INFINITY;
            const float nm = none ? 0.f : -M[hf];
            // (at most kSlack; 2^-300 of anything is 0)
            const int up = (int)__builtin_fmaxf(none ? -300.f : M[hf] - ref, -300.f);
            float sum = 0.f;
#pragma unroll
            for (int kt = 4 * hf; kt < 4 * hf + 4; ++kt) {
                float e[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][r], c[hf], nm));
                    sum += e[r];
                }
                s16x2 word = {};
                word = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(word, e[0], e[1], 0x1p-8f, false);
                word = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(word, e[2], e[3], 0x1p-8f, true);
                pk[kt] = __builtin_bit_cast(int, word);
            }
            ell += __builtin_amdgcn_ldexpf(sum, up);
            // the group's scale, and the 2^8 of the codes taken back
            sb[hf] = (uint32_t)max(127 - 8 + lent[hf] + up, 0);
        }
        // group j of the visit's four gets its scale from lane group j: 0 and 1 are the
        // first half's of lane groups 0, 1 and 2, 3; 2 and 3 the second half's
        const auto sw = __builtin_amdgcn_permlane32_swap(sb[0], sb[1], false, false);
        const int scale_b = (int)(g & 1 ? sw[1] : sw[0]);
        // ---- O^T += V^T P^T (this visit's V is older than the next one's K) ----
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NI) : "memory");
        auto v_read = [&](int dt) __attribute__((always_inline)) {
            i32x8 av;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const i32x2 t = read_tr8(vst + (v_lane ^ (uint32_t)(dt << 4)) + (64 * (u / 2) + 8 * (u % 2)) * D);
                av[2 * u] = t[0];
                av[2 * u + 1] = t[1];
            }
            return av;
        };
        // Where some rows see keys that others do not, a NaN of V must not reach the others
        // by way of 0 times NaN: it makes NaN of the sums of the rows that see it, and goes.
        if (t0 + kVisit - 1 > pos_min && pos_min + 1 < seen && holds_nan(vst, STAGE, lane)) {
            i32x8 see;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
                see[kt] = ones(pos - t0 - 64 * (kt / 4) - 16 * g - 4 * (kt % 4) + 1);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const f32x4 hits = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(nan_ones(v_read(dt)), see, f32x4{}, 0, 0, 0, 127, 0, 127);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    o[dt][r] = hits[r] > 0.f ? __builtin_nanf("") : o[dt][r];
            }
            clear_nans(vst, STAGE, lane);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const i32x8 av = v_read(dt);
            o[dt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, pk, o[dt], 0, 0, 0, sa, 0, scale_b);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        issue_v(v + NW);
    }

    // ---- the waves' (O, l) at the row's largest reference ----
    ell += __shfl_xor(ell, 16, 64);
    ell += __shfl_xor(ell, 32, 64);
    // (the last, empty loads write zeros into the stages: they have to have landed)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (g == 0) {
        lsh[w][n] = ell;
        msh[w][n] = ref;
    }
    __syncthreads();
    float m = msh[0][n];
#pragma unroll
    for (int i = 1; i < NW; ++i)
        m = fmax_f(m, msh[i][n]);
    const int down = shift_of(ref, m);
    float* const mw = reinterpret_cast<float*>(lds) + (w * TR + n) * MS;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            x[r] = __builtin_amdgcn_ldexpf(o[dt][r], down);
        *reinterpret_cast<f32x4*>(mw + 16 * dt + 4 * g) = x;
    }
    __syncthreads();
    const float* mb = reinterpret_cast<const float*>(lds);
    const size_t stride = (size_t)TR * (D + 2);
    float* const part = whole ? nullptr
                              : p.ws + ((((size_t)b * p.cache.Hkv + hk) * p.tiles + tile) * p.ranges + range) * stride;
    for (int e = tid; e < TR * D / 4; e += 256) {
        const int rr = e / (D / 4), piece = e % (D / 4);
        if (row0 + rr >= rows)
            continue;
        f32x4 acc = *reinterpret_cast<const f32x4*>(mb + rr * MS + 4 * piece);
        float mm = msh[0][rr];
#pragma unroll
        for (int i = 1; i < NW; ++i)
            mm = fmax_f(mm, msh[i][rr]);
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i)
            l += msh[i][rr] == -INFINITY ? 0.f : lsh[i][rr] * __builtin_amdgcn_exp2f(msh[i][rr] - mm);
#pragma unroll
        for (int i = 1; i < NW; ++i) {
            const f32x4 t = *reinterpret_cast<const f32x4*>(mb + (i * TR + rr) * MS + 4 * piece);
#pragma unroll
            for (int c = 0; c < 4; ++c)
                acc[c] += t[c];
        }
        if (whole) {
            write_row<D>(p, s, hk, row0 + rr, piece, acc, l, 1.f / l, mm);
        } else {
            *reinterpret_cast<f32x4*>(part + rr * D + 4 * piece) = acc;
            if (piece == 0) {
                part[TR * D + rr] = l;
                part[TR * (D + 1) + rr] = mm;
            }
        }
    }
}

}  // namespace attn
