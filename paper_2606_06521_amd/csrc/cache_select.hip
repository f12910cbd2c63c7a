// Choice of pages: for a run of new tokens and a KV head the pages whose bounds allow the
// largest scores.
//
// A key k of a page lies between lo and hi in every channel, so q k <= sum_c max(q lo, q hi)
// = q+ hi + q- lo with q+ and q- the positive and negative parts of q: two matrix products.
// q is rounded to whole numbers up to 127 on a power of two of its row, lo and hi are codes
// that are multiples of 1/2 up to 448: sums of 128 channels stay below 2^24 of these halves,
// so the bf16 matrix cores' FP32 sums are exact in any order and the choice does not depend on it.
//
// One workgroup per list.  Its waves load a tile of 32 pages each, in whole lines, and stage it in
// LDS; then they share out the products of these tiles and the tiles of 32 rows: S = Q B^T with
// lane n holding 16 rows' scores of page n, so that a page's largest is taken within the lane,
// and over the tiles of rows by a maximum in LDS of keys that order as the scores do (whole
// numbers: the result does not depend on the order of the waves).  The choice is a radix choice:
// a histogram over the range of the keys, again over a digit that more than 64 pages share, and
// the rank of those that are left.
//
// What bounds it: single tokens a chain of loads (offsets, length, page numbers, bounds) and
// the choice, 6.0 us for 4 sequences of 777 keys; 8.4 for 16 x 8 heads x 256 pages of 128 channels
// (8.4 MB of bounds; pairwise ranks in the place of the histograms 11.3).  Few lists of many pages are scored by several
// workgroups a list and chosen by a second launch: 8 lists x 2047 pages 11.0 us, by one workgroup
// a list 32.3.  A chunk (64 runs of 32 tokens x 4 heads on 128 pages, 8 heads) 13.5 us (26.4 with bounds
// loaded by the lanes that multiply them, which reads every line 8 times), in phases: of a wave's 25 thousand
// cycles the vector unit, which two waves share, is busy for 49 %, the matrix core for 16 %, LDS for 10 %, and
// a wave waits for 34 %; q (16.8 MB, 3 us at the rate of memory) comes from HBM once, by lanes that
// read each line eight times.
#include "cache_common.hpp"

#include <algorithm>
#include <type_traits>

namespace attn {

namespace {

// Orders as the numbers do, as unsigned; above 0 and below the largest.
__device__ inline uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exponents up to here stay away from FP32's ends and, with those of a page's scale up to 96 - this, from
// the bounds of their sum.
constexpr int kPlain = 60;

// Up to here the keys leave room in LDS for several workgroups.
constexpr int kFewPages = 2048;

// Pages that a workgroup of a split call scores at most.
constexpr int kPartPages = 1024;

// What the wave's lanes wrote to LDS is read by its others.
__device__ inline void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The tokens of a run.
__device__ inline Seq run_of(const SelectParams& p, int b, int run)
{
    Seq s = uniform(sequence(p.bt, b, p.max_len));
    s.first += run * p.run;
    s.pos0 += run * p.run;
    s.n = min(max(s.n - run * p.run, 0), p.run);
    return s;
}

// Blocks that its last token sees a key of.
__device__ inline int seen_blocks(const SelectParams& p, const Seq& s, int page)
{
    const int seen = s.n > 0 ? last_key(s.pos0 + s.n - 1, p.causal, s.len) + 1 : 0;
    return (max(seen, 0) + page - 1) / page;
}

// A lane's value with another's of its row of 16, by a cross-lane move.
template <int CTRL, int ROWS = 15>
__device__ inline uint32_t moved(uint32_t x, uint32_t none)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 15, false);
}

// Over the wave, in all lanes (`f` of two values; in rows of 16 by rotations).
template <class F>
__device__ inline uint32_t over_wave(uint32_t x, F f)
{
    x = f(x, moved<0x128>(x, 0));
    x = f(x, moved<0x124>(x, 0));
    x = f(x, moved<0x122>(x, 0));
    x = f(x, moved<0x121>(x, 0));
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return f(b[0], b[1]);
}

// Sum of the lanes up to this one (shifts in rows of 16, then the rows' sums).
__device__ inline uint32_t sum_up_to(uint32_t x)
{
    x += moved<0x111>(x, 0);
    x += moved<0x112>(x, 0);
    x += moved<0x114>(x, 0);
    x += moved<0x118>(x, 0);
    x += moved<0x142, 10>(x, 0);
    x += moved<0x143, 12>(x, 0);
    return x;
}

// What a choice keeps in LDS beside the keys.
struct Scratch {
    __attribute__((aligned(16))) int hist[256];
    uint32_t near_key[64], lowest, highest;
    int always, near, sums[8][2];
    __device__ inline void clear(int threads)
    {
        for (int i = threadIdx.x; i < 256; i += threads)
            hist[i] = 0;
        if (threadIdx.x == 0) {
            lowest = ~0u;
            highest = 0;
            always = near = 0;
        }
    }
};

// What NW waves (one: the first of the workgroup, by itself) wrote to LDS is read by each of them.
template <int NW>
__device__ inline void shared_fence()
{
    if constexpr (NW > 1)
        lds_barrier();
    else
        wave_fence();
}

// The key `floor` of the last page that is taken, and how many of its equals are (`left`).  lo, hi, must: the
// lane's least and largest key that is not forced, the wave's number of those that are (all ones in k).
template <int NW, int R>
__device__ inline void find_floor(Scratch& sc, const uint32_t (&k)[R], uint32_t lo, uint32_t hi, int must, int take, uint32_t& floor, int& left)
{
    const int tid = threadIdx.x, lane = tid & 63;
    lo = over_wave(lo, [](uint32_t a, uint32_t b) { return min(a, b); });
    hi = over_wave(hi, [](uint32_t a, uint32_t b) { return max(a, b); });
    if (lane == 0) {
        atomicMin(&sc.lowest, lo);
        atomicMax(&sc.highest, hi);
        if (must > 0)
            atomicAdd(&sc.always, must);
    }
    shared_fence<NW>();

    // `lo` .. `hi` holds the keys that are not decided yet; `before` pages come before them (those
    // that are always taken, and keys above hi)
    lo = sc.lowest;
    hi = max(sc.highest, lo);
    int before = sc.always;
    for (;;) {
        const int shift = max(32 - 8 - (hi == lo ? 32 : __builtin_clz(hi - lo)), 0);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (k[r] >= lo && k[r] <= hi && k[r] != ~0u)
                atomicAdd(&sc.hist[(k[r] - lo) >> shift], 1);
        shared_fence<NW>();
        // the highest digit at which the list is full (every wave by itself)
        int c[4], sum = 0;
        const i32x4 bins = *reinterpret_cast<const i32x4*>(&sc.hist[4 * (63 - lane)]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            c[j] = bins[3 - j];
            sum += c[j];
        }
        int ahead = before + (int)sum_up_to((uint32_t)sum) - sum;
        int digit = -1, at = 0, count = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (digit < 0 && ahead < take && ahead + c[j] >= take) {
                digit = 255 - 4 * lane - j;
                at = ahead;
                count = c[j];
            }
            ahead += c[j];
        }
        const uint64_t who = __ballot(digit >= 0);
        if (who == 0) {
            // (the pages that are always taken fill the list, or there are no more than it takes)
            floor = before >= take ? ~0u : 0u;
            break;
        }
        const int from = __builtin_ctzll(who);
        digit = __builtin_amdgcn_readlane(digit, from);
        before = __builtin_amdgcn_readlane(at, from);
        count = __builtin_amdgcn_readlane(count, from);
        lo += (uint32_t)digit << shift;
        hi = min(hi, lo + ((1u << shift) - 1));
        if (shift == 0) {               // all of them equal
            floor = lo;
            left = take - before;
            break;
        }
        if (count <= 64) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (k[r] >= lo && k[r] <= hi && k[r] != ~0u)
                    sc.near_key[atomicAdd(&sc.near, 1)] = k[r];
            shared_fence<NW>();
            const uint32_t mine = lane < count ? sc.near_key[lane] : 0u;
            int above = 0, equal = 0;
            for (int i = 0; i < count; ++i) {
                const uint32_t o = __builtin_amdgcn_readlane(mine, i);
                above += o > mine;
                equal += o == mine;
            }
            // (lanes of equal keys say the same)
            const uint64_t last = __ballot(lane < count && above < take - before && above + equal >= take - before);
            const int l = __builtin_ctzll(last);
            floor = __builtin_amdgcn_readlane(mine, l);
            left = take - before - __builtin_amdgcn_readlane(above, l);
            break;
        }
        shared_fence<NW>();
        for (int i = tid; i < 256; i += 64 * NW)
            sc.hist[i] = 0;
        shared_fence<NW>();
    }
}

// The `take` largest of nb keys (0: no page; those that are forced: always), equal ones from the
// first on, as an ascending list.  A lane holds keys i0 + 64 r + lane of its wave's part, r < R.
template <int NW, int R, class K, class F>
__device__ inline void choose_of(Scratch& sc, K key, int32_t* list, int take, int nb, F forced)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i0 = w * R * 64;
    uint32_t k[R], lo = ~0u, hi = 0;
    int must = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = i0 + 64 * r + lane;
        k[r] = i < nb ? key(i) : 0u;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool always = k[r] != 0 && forced(i0 + 64 * r + lane);
        must += __builtin_popcountll(__ballot(always));
        lo = k[r] != 0 && !always ? min(lo, k[r]) : lo;
        hi = always ? hi : max(hi, k[r]);
        k[r] = always ? ~0u : k[r];
    }
    uint32_t floor = 0;
    int left = 0;
    if (nb > take)          // (else all that there are)
        find_floor<NW, R>(sc, k, lo, hi, must, take, floor, left);

    // ---- their places, in order ----
    // (floor = all ones: only those that are always taken)
    uint64_t up[R], eq[R];
    int above = 0, equal = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        up[r] = __ballot(k[r] > floor || k[r] == ~0u);
        eq[r] = __ballot(k[r] == floor && k[r] != 0 && k[r] != ~0u);
        above += __builtin_popcountll(up[r]);
        equal += __builtin_popcountll(eq[r]);
    }
    if (lane == 0) {
        sc.sums[w][0] = above;
        sc.sums[w][1] = equal;
    }
    shared_fence<NW>();
    int sure = 0, ties = 0, all = 0, all_ties = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const int a = sc.sums[i][0], e = sc.sums[i][1];
        sure += i < w ? a : 0;
        ties += i < w ? e : 0;
        all += a;
        all_ties += e;
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int t = ties + __builtin_popcountll(eq[r] & below);
        if ((up[r] >> lane & 1) || ((eq[r] >> lane & 1) && t < left))
            list[sure + __builtin_popcountll(up[r] & below) + min(t, left)] = i0 + 64 * r + lane;
        sure += __builtin_popcountll(up[r]);
        ties += __builtin_popcountll(eq[r]);
    }
    for (int i = all + min(all_ties, left) + tid; i < take; i += 64 * NW)
        list[i] = -1;
}

template <int NW, int MOST, class K, class F>
__device__ inline void choose(Scratch& sc, K key, int32_t* list, int take, int nb, F forced)
{
    constexpr int WAVES = 64 * NW;
    if (nb <= 256) {
        if (threadIdx.x < 64)
            choose_of<1, 4>(sc, key, list, take, nb, forced);
        return;
    }
    if (nb <= WAVES)
        return choose_of<NW, 1>(sc, key, list, take, nb, forced);
    if constexpr (MOST > WAVES) {
        if (nb <= 4 * WAVES)
            return choose_of<NW, 4>(sc, key, list, take, nb, forced);
        if constexpr (MOST > 4 * WAVES)
            choose_of<NW, (MOST + WAVES - 1) / WAVES>(sc, key, list, take, nb, forced);
    }
}

template <int D, bool E4M3, int TR, int NW, int MOST, bool SCORES>
__global__ void __launch_bounds__(64 * NW) select_kernel(SelectParams p, int page)
{
    constexpr int LG = 64 / TR;             // lanes of a row or page: each takes every LG-th piece
    constexpr int NI = D / 16 / LG;         // 16-byte pieces of a row and lane
    constexpr int NR = TR * TR / 64;        // rows of a lane's scores
    typedef float acc_t __attribute__((ext_vector_type(NR)));
    constexpr int CB = 2 * D / 16;          // 16-byte pieces of a page's bounds
    constexpr int NL = 32 * CB / 64;        // loads of a tile
    __shared__ __attribute__((aligned(16))) uint8_t stage[NW][32 * 2 * D];
    __shared__ uint32_t key[MOST];
    __shared__ int scale_of[NW][32], row_e[NW][TR], row_last[NW][TR];
    __shared__ Scratch sc;

    const int units = p.bt.B * p.cache.Hkv * p.runs * (SCORES ? p.parts : 1), per_xcd = (units + kNumXcd - 1) / kNumXcd;
    const int slot = (int)(blockIdx.x / kNumXcd);
    int unit = (int)(blockIdx.x % kNumXcd) * per_xcd + slot;
    if (slot >= per_xcd || unit >= units)
        return;
    // the part of the pages that is looked at here
    const int offset = SCORES ? unit % p.parts * p.part : 0;
    unit = SCORES ? unit / p.parts : unit;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int run = unit % p.runs, hk = unit / p.runs % p.cache.Hkv, b = unit / p.runs / p.cache.Hkv;
    // (a page behind the last key that is seen may be any: its bounds are not used)
    auto page_at = [&](int block) __attribute__((always_inline)) { return page_of(p.bt, p.cache.n_pages, b, offset + block); };
    int pid = page_at(32 * w + (lane & 31));
    const Seq s = run_of(p, b, run);
    const int n = lane & (TR - 1), h = lane / TR;       // row or page of a tile, and the lane of it
    const int rows = s.n * p.gr.G, row_tiles = (rows + TR - 1) / TR;
    const int blocks = seen_blocks(p, s, page);
    const int nb = SCORES ? min(max(blocks - offset, 0), p.part) : blocks;
    int32_t* const list = p.blocks + (((int64_t)b * p.runs + run) * p.cache.Hkv + hk) * p.take;
    auto forced = [&](int block) __attribute__((always_inline)) { return block < p.n_first || block >= blocks - p.n_last; };

    // ---- scores ----
    // (waves per tile of pages: as many as there are tiles of rows)
    int by_rows = 1;
    while (by_rows < NW && by_rows < row_tiles)
        by_rows *= 2;
    const int wr = w & (by_rows - 1), wc = w / by_rows, by_pages = NW / by_rows;
    // piece c of a page's bounds lies at c ^ swz(page): the 32 pages' same pieces in distinct banks
    auto swz = [](int i) __attribute__((always_inline)) { return D == 128 ? i & 15 : i >> 1 & 7; };
    struct Pages {
        i32x4 x[NL];
        int scale;
    };
    auto load = [&](int pid) __attribute__((always_inline)) {
        Pages r;
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int i = 64 / CB * j + lane / CB, of = __shfl(pid, i, 64);
            const uint8_t* const from = p.bounds + ((size_t)max(of, 0) * p.cache.Hkv + hk) * (2 * D);
            r.x[j] = of < 0 ? i32x4{} : *reinterpret_cast<const i32x4*>(from + 16 * (lane % CB ^ swz(i)));
        }
        // (of the lane's page of the tile)
        r.scale = pid < 0 ? -1 : p.cache.ks[(size_t)pid * p.cache.Hkv + hk];
        return r;
    };
    for (int i = tid; i < nb; i += 64 * NW)
        key[i] = 0;
    sc.clear(64 * NW);
    lds_barrier();
    for (int rt = 0; rt < row_tiles; rt += by_rows) {
        bf16x8 qp[2 * NI], qn[2 * NI];
        int row0 = TR * (rt + wr);
        const bool works = row0 < rows;
        row0 = works ? row0 : 0;
        const int row = min(row0 + n, rows - 1), i = p.gr.token(row);
        const int64_t at = (int64_t)(s.first + i) * p.q.st + (int64_t)(hk * p.gr.G + (row - i * p.gr.G)) * p.q.sh;
        // fragment 2 i + e of lane h: channels 16 (LG i + h) + 8 e on
#pragma unroll
        for (int j = 0; j < 2 * NI; ++j)
            qp[j] = load_q8<E4M3>(p.q.data, at + 16 * (LG * (j / 2) + h) + 8 * (j % 2));
        Pages next = load(pid);
        pid = page_at(32 * (NW + w) + (lane & 31));
        asm volatile("" ::: "memory");      // (the loads are under way from here on)
        bool plain;             // no exponent near its bounds
        int first_last;         // what all rows see
        {
            typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
            typedef int16_t s16x8 __attribute__((ext_vector_type(8)));
            u16x8 m = {};
#pragma unroll
            for (int j = 0; j < 2 * NI; ++j)
                m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x8, qp[j]) & (u16x8)((uint16_t)0x7FFF));
            uint16_t top = 0;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                top = m[c] > top ? m[c] : top;
#pragma unroll
            for (int off = 32; off >= TR; off >>= 1)
                top = (uint16_t)max((int)top, __shfl_xor((int)top, off, 64));
            const bool good = top < 0x7F80;
            const float f = __uint_as_float((uint32_t)top << 16);
            // least e with f <= 127 2^e: 127 = 0.9921875 * 2^7
            int e = __builtin_amdgcn_frexp_expf(f) - 7 + (__builtin_amdgcn_frexp_mantf(f) > 0.9921875f ? 1 : 0);
            e = good && top != 0 ? e : 0;
            // (a row that is not finite sees no page; one past the last is the last again)
            const int last = good ? last_key(s.pos0 + i, p.causal, s.len) : -1;
            first_last = (int)over_wave((uint32_t)(last + 1), [](uint32_t a, uint32_t b) { return min(a, b); }) - 1;
            plain = __ballot(abs(e) > kPlain) == 0;
            // the whole numbers times 2^e (past kPlain: 2^kPlain): a sum with 3 2^(e + 22) leaves a
            // multiple of 2^e, rounded to even
            const int scaled = min(max(e, -kPlain), kPlain);
            const float lift = __builtin_amdgcn_ldexpf(0x1.8p23f, scaled);
            if (!plain) {
#pragma unroll
                for (int j = 0; j < 2 * NI; ++j)
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        qp[j][c] = (__bf16)__builtin_amdgcn_ldexpf((float)qp[j][c], scaled - e);
            }
#pragma unroll
            for (int j = 0; j < 2 * NI; ++j) {
                bf16x8 y;
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    y[c] = (__bf16)(((float)qp[j][c] + lift) - lift);
                // its negative part and the rest
                const s16x8 bits = __builtin_bit_cast(s16x8, y), neg = bits & (bits >> 15);
                qn[j] = __builtin_bit_cast(bf16x8, neg);
                qp[j] = __builtin_bit_cast(bf16x8, (s16x8)(bits ^ neg));
            }
            wave_fence();
            if (h == 0) {
                row_e[w][n] = e;
                row_last[w][n] = last;
            }
            wave_fence();
        }
        for (int b0 = 0; b0 < nb; b0 += 32 * NW) {
#pragma unroll
            for (int j = 0; j < NL; ++j)
                *reinterpret_cast<i32x4*>(&stage[w][1024 * j + 16 * lane]) = next.x[j];
            if (lane < 32)
                scale_of[w][lane] = next.scale;
            if (by_rows > 1)
                lds_barrier();
            else
                wave_fence();
            if (b0 + 32 * (NW + w) < nb) {
                next = load(pid);
                pid = page_at(b0 + 32 * (2 * NW + w) + (lane & 31));
            }
            for (int c = wc; works && c < NW && b0 + 32 * c < nb; c += by_pages)
#pragma unroll
                for (int part = 0; part < 32 / TR; ++part) {
                    const int slot = TR * part + n;                 // of the staged pages
                    acc_t acc = {};
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int j = 0; j < NI; ++j) {
                            const int piece = half * (D / 16) + LG * j + h;
                            const i32x4 v = *reinterpret_cast<const i32x4*>(&stage[c][slot * (2 * D) + 16 * (piece ^ swz(slot))]);
                            const bf16x8 k0 = widen((uint32_t)v[0], (uint32_t)v[1]), k1 = widen((uint32_t)v[2], (uint32_t)v[3]);
                            if constexpr (TR == 32) {
                                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(half ? qp[2 * j] : qn[2 * j], k0, acc, 0, 0, 0);
                                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(half ? qp[2 * j + 1] : qn[2 * j + 1], k1, acc, 0, 0, 0);
                            } else {
                                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(half ? qp[2 * j] : qn[2 * j], k0, acc, 0, 0, 0);
                                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(half ? qp[2 * j + 1] : qn[2 * j + 1], k1, acc, 0, 0, 0);
                            }
                        }
                    const int block = b0 + 32 * c + slot, byte = scale_of[c][slot], scale = max(byte, 0) - 127;
                    float best = -INFINITY;
                    const int from = (offset + block) * page;
                    const bool all_see = __ballot(from > first_last) == 0;
                    if (plain && all_see && __ballot(abs(scale) > 96 - kPlain) == 0) {
#pragma unroll
                        for (int r = 0; r < NR; ++r)
                            best = fmax_f(best, acc[r]);
                        best = __builtin_amdgcn_ldexpf(best, scale);
                    } else {
#pragma unroll
                        for (int r = 0; r < NR; ++r) {
                            const int at = 8 * (r / 4) + 4 * h + r % 4, e = row_e[w][at];
                            const int up = min(max(e + scale, -96), 96) - min(max(e, -kPlain), kPlain);
                            const float u = __builtin_amdgcn_ldexpf(acc[r], up);
                            best = fmax_f(best, from <= row_last[w][at] ? u : -INFINITY);
                        }
                    }
                    best = halves_max(best);
                    if constexpr (TR == 16)
                        best = fmax_f(best, __shfl_xor(best, 16, 64));
                    if (h == 0 && byte >= 0 && block < nb) {
                        const uint32_t k = key_of(best);
                        // (a single tile of rows: one wave has the page, once)
                        if (by_rows > 1)
                            atomicMax(&key[block], k);
                        else
                            key[block] = k;
                    }
                }
            if (by_rows > 1)
                lds_barrier();
            else
                wave_fence();
        }
        pid = page_at(32 * w + (lane & 31));
    }
    lds_barrier();
    if constexpr (SCORES) {
        uint32_t* const to = p.keys + (int64_t)unit * p.most + offset;
        for (int i = tid; i < nb; i += 64 * NW)
            to[i] = key[i];
    } else {
        choose<NW, MOST>(sc, [&](int i) __attribute__((always_inline)) { return key[i]; }, list, p.take, nb, forced);
    }
}

template <int NW>
__global__ void __launch_bounds__(64 * NW) pick_kernel(SelectParams p, int page)
{
    __shared__ Scratch sc;
    const int unit = (int)blockIdx.x, run = unit % p.runs, hk = unit / p.runs % p.cache.Hkv, b = unit / p.runs / p.cache.Hkv;
    const Seq s = run_of(p, b, run);
    const int nb = seen_blocks(p, s, page);
    int32_t* const list = p.blocks + (((int64_t)b * p.runs + run) * p.cache.Hkv + hk) * p.take;
    auto forced = [&](int block) __attribute__((always_inline)) { return block < p.n_first || block >= nb - p.n_last; };
    sc.clear(64 * NW);
    lds_barrier();
    const uint32_t* const from = p.keys + (int64_t)unit * p.most;
    choose<NW, kMaxChoice>(sc, [&](int i) __attribute__((always_inline)) { return from[i]; }, list, p.take, nb, forced);
}

}  // namespace

// Few lists of many pages: parts of them by workgroups of their own, then a launch for the choice.
SelectPlan select_plan(int64_t lists, int most)
{
    SelectPlan pl{1, most, 0};
    if (lists > 0 && most > (lists > 64 ? 512 : 256) && lists <= 128) {
        const int64_t want = std::min<int64_t>(512 / lists, (most + 127) / 128);
        pl.part = (int)std::min<int64_t>(((most + want - 1) / want + 127) / 128 * 128, kPartPages);
        pl.parts = (most + pl.part - 1) / pl.part;
        pl.bytes = (size_t)lists * most * sizeof(uint32_t);
    }
    return pl;
}

hipError_t launch_cache_select(SelectParams p, const SelectPlan& pl, int d, int page, bool e4m3, hipStream_t s)
{
    p.parts = pl.parts;
    p.part = pl.part;
    p.most = (p.max_len + page - 1) / page;
    const __int128 units = (__int128)p.bt.B * p.cache.Hkv * p.runs;
    unsigned grid;
    const hipError_t e = grid_of((units * pl.parts + kNumXcd - 1) / kNumXcd * kNumXcd, 512, grid);
    if (e != hipSuccess)
        return e;
    auto go = [&](auto kern, int nw) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * nw), 0, s, p, page);
        return hipGetLastError();
    };
    const bool low = (int64_t)p.run * p.gr.G <= 16;
    auto of_type = [&](auto wide, auto type, auto rows) {
        constexpr int D = decltype(wide)::value, TR = decltype(rows)::value;
        constexpr bool E = decltype(type)::value;
        if (pl.bytes > 0)
            return go(select_kernel<D, E, TR, 4, kPartPages, true>, 4);
        if (p.most > kFewPages)
            return go(select_kernel<D, E, TR, 8, kMaxChoice, false>, 8);
        return units > 256 ? go(select_kernel<D, E, TR, 4, kFewPages, false>, 4) : go(select_kernel<D, E, TR, 8, kFewPages, false>, 8);
    };
    auto of_rows = [&](auto wide, auto type) {
        return low ? of_type(wide, type, std::integral_constant<int, 16>{}) : of_type(wide, type, std::integral_constant<int, 32>{});
    };
    auto of_size = [&](auto wide) { return e4m3 ? of_rows(wide, std::true_type{}) : of_rows(wide, std::false_type{}); };
    hipError_t r = d == 64 ? of_size(std::integral_constant<int, 64>{}) : of_size(std::integral_constant<int, 128>{});
    if (r == hipSuccess && pl.bytes > 0) {
        hipLaunchKernelGGL(pick_kernel<8>, dim3((unsigned)units), dim3(512), 0, s, p, page);
        r = hipGetLastError();
    }
    return r;
}

}  // namespace attn
