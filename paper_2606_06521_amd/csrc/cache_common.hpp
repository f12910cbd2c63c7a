// The KV cache's kernels: launch parameters, the sequences and pages of a batch,
// element types.
#pragma once

#include "attn_common.hpp"

namespace attn {

// element types (the values of ATTN_TYPE_*)
constexpr int kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2, kTypeE4m3 = 3;

// Keys per visit of the attention kernels.
constexpr int kVisit = 128;

// The batch, as the device reads it.  Nothing in lens, cu or pages is trusted:
// whatever they hold, no access leaves the arrays.
struct Batch {
    const int32_t* pages;   // [B][W]
    const int32_t* lens;    // [B]
    const int32_t* cu;      // [B + 1], or null: `uniform` tokens each
    int B, W, T, max_q, uniform;
};

struct Cache {
    uint8_t* k;
    uint8_t* v;
    uint8_t* ks;
    uint8_t* vs;
    int n_pages, Hkv;
};

// Packed heads [T][H][d]: element strides.
struct Heads {
    void* data;
    int64_t st, sh;
};

struct Rotation {
    const float* table;          // [n_pos][rot / 2][2], null: no rotation
    const int32_t* positions;    // null: the position in the sequence
    int n_pos, rot, layout;      // layout 0: halves, 1: interleaved
};

// Sequence b: the keys there are (its length, at most max_len), its new tokens
// [first, first + n) of the call (at most max_q, inside [0, T)), the position of the
// first of them (by its whole length: it may lie before 0 or past the keys).
struct Seq {
    int len, first, n, pos0;
};

__device__ inline Seq sequence(const Batch& bt, int b, int max_len)
{
    Seq s;
    const int whole = max(bt.lens[b], 0);
    s.len = min(whole, max_len);
    int n;
    if (bt.cu) {
        const int c0 = bt.cu[b], c1 = bt.cu[b + 1];
        s.first = min(max(c0, 0), bt.T);
        n = min(max(c1, s.first), bt.T) - s.first;
    } else {
        s.first = b * bt.uniform;
        n = bt.uniform;
    }
    s.pos0 = whole - n;
    s.n = min(n, bt.max_q);
    return s;
}

// The same in scalar registers, for a sequence that all lanes share.
__device__ inline Seq uniform(const Seq& s)
{
    return {__builtin_amdgcn_readfirstlane(s.len), __builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.n),
            __builtin_amdgcn_readfirstlane(s.pos0)};
}

// The last key that the query at position `at` sees of `len` (below 0: none; a token before
// position 0 sees none, causal or not).
__device__ inline int last_key(int at, int causal, int len)
{
    return at < 0 ? -1 : causal ? min(at, len - 1) : len - 1;
}

// Query rows of a (sequence, KV head): row R is head R % G of token R / G.
struct Group {
    int G;
    uint32_t mul;           // ceil(2^32 / G) (G = 1: 0): exact for R G < 2^32
    __device__ inline int token(int R) const { return mul ? (int)__umulhi((uint32_t)R, mul) : R; }
};

inline Group group_of(int G) { return {G, G == 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + G - 1) / G)}; }

// Page of a sequence's block, -1 if there is none.
__device__ inline int page_of(const Batch& bt, int n_pages, int b, int block)
{
    const int p = block < bt.W ? bt.pages[(size_t)b * bt.W + block] : -1;
    return (uint32_t)p < (uint32_t)n_pages ? p : -1;
}

// ---- E4M3 blocks ----

// Least e >= -127 with amax <= 448 * 2^e (amax >= 0 and finite).
__device__ inline int block_exponent(float amax)
{
    if (amax == 0.f)
        return -127;
    const int t = __builtin_amdgcn_frexp_expf(amax);
    const float f = __builtin_amdgcn_frexp_mantf(amax);   // [0.5, 1): 448 = 0.875 * 2^9
    return max(t - 9 + (f > 0.875f ? 1 : 0), -127);
}

// Four values to E4M3 bytes (round to nearest even; |x| <= 448 or NaN).
__device__ inline uint32_t to_e4m3(float a, float b, float c, float d)
{
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

__device__ inline void from_e4m3(uint32_t w, float* x)
{
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}

// Factor of a block's scores, c 2^(byte - 127), kept off 0 and infinity: a masked key's
// -inf stays one, and a score of 0 too.
__device__ inline float score_factor(float c, int byte)
{
    return __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(c, byte - 127), 0x1p-149f, 0x1.fffffep127f);
}

// Binary exponent of 2^(from - to), from <= to powers of two of a row's sums: applied with
// ldexp, since as a number it underflows where a sum of large values does not (a sum of 2^128
// at most: 2^-300 of it is 0).  from = -inf: a sum of 0.
__device__ inline int shift_of(float from, float to)
{
    return from == to || from == -INFINITY ? 0 : (int)__builtin_fmaxf(from - to, -300.f);
}

// What of V's scale byte goes into the scale of P: a matrix core's scale ends at 2^-127, a group's
// power of two relative to the row's does not (down to -119 - this it is exact; up to kSlack
// the byte stays below 255).
__device__ inline int lent_scale(int vbyte) { return min(vbyte, 119); }

// ---- eight consecutive values of an element type ----

template <int TYPE>
__device__ inline void load8(const void* base, int64_t i, float* x)
{
    if constexpr (TYPE == kTypeF32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + i);
        const f32x4 a = p[0], b = p[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = a[j];
            x[4 + j] = b[j];
        }
    } else {
        const i32x4 w = *reinterpret_cast<const i32x4*>(static_cast<const uint16_t*>(base) + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t u = (uint32_t)w[j];
            if constexpr (TYPE == kTypeBf16) {
                x[2 * j] = __uint_as_float(u << 16);
                x[2 * j + 1] = __uint_as_float(u & 0xFFFF0000u);
            } else {
                x[2 * j] = (float)__builtin_bit_cast(_Float16, (uint16_t)u);
                x[2 * j + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(u >> 16));
            }
        }
    }
}

template <int TYPE>
__device__ inline void store8(void* base, int64_t i, const float* x)
{
    if constexpr (TYPE == kTypeF32) {
        f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(base) + i);
        p[0] = f32x4{x[0], x[1], x[2], x[3]};
        p[1] = f32x4{x[4], x[5], x[6], x[7]};
    } else {
        i32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (TYPE == kTypeBf16)
                w[j] = (int)((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * j]) |
                             (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * j + 1]) << 16);
            else
                w[j] = (int)((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * j]) |
                             (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * j + 1]) << 16);
        }
        *reinterpret_cast<i32x4*>(static_cast<uint16_t*>(base) + i) = w;
    }
}

namespace {

// Buffer over `bytes` bytes at a uniform address (what lies behind them reads as
// 0), as the instruction takes it.
__device__ inline i32x4 bytes_buffer(const uint8_t* base, int bytes)
{
    const uint64_t a = (uint64_t)(uintptr_t)base;
    return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)a), __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xFFFF),
                 __builtin_amdgcn_readfirstlane(bytes), 0x00027000};
}

// 16 bytes per lane from a buffer straight into LDS: lane i's to dst + 16 i.  As
// inline assembly, so that the compiler does not make every LDS read wait for the
// loads in flight (it cannot tell the stages apart); the kernel waits by vmcnt.
__device__ inline void load_lds16(i32x4 buf, uint32_t voff, uint32_t soff, const uint8_t* dst)
{
    const uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)dst;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(at)), "v"(voff), "s"(buf),
                   "s"(__builtin_amdgcn_readfirstlane(soff))
                 : "memory");
}

// The same from an address per lane.
__device__ inline void load_lds16(const uint8_t* src, const uint8_t* dst)
{
    const uint32_t at = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t*)dst;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(at)), "v"(src)
                 : "memory");
}

__device__ inline i32x2 read_tr8(const uint8_t* p)
{
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)(p));
}

// Eight E4M3 codes as bf16 (exact).
__device__ inline bf16x8 widen(uint32_t a, uint32_t b)
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    const bf2 x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const bf2 x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return bf16x8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}

// Eight channels of a query row as bf16.
template <bool E4M3>
__device__ inline bf16x8 load_q8(const void* q, int64_t at)
{
    if constexpr (E4M3) {
        const i32x2 w = *reinterpret_cast<const i32x2*>(static_cast<const uint8_t*>(q) + at);
        return widen((uint32_t)w[0], (uint32_t)w[1]);
    } else {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<const i32x4*>(static_cast<const uint16_t*>(q) + at));
    }
}

}  // namespace

// The NaN codes of a word of four: 0x80 in their bytes.
__device__ inline uint32_t nan_bytes(uint32_t w)
{
    return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// Whether `bytes` (a multiple of 1024) of LDS hold a NaN code; the wave looks at all of them.
__device__ inline bool holds_nan(const uint8_t* p, int bytes, int lane)
{
    uint32_t any = 0;
    for (int i = 16 * lane; i < bytes; i += 1024) {
        const i32x4 x = *reinterpret_cast<const i32x4*>(p + i);
        any |= nan_bytes(x[0]) | nan_bytes(x[1]) | nan_bytes(x[2]) | nan_bytes(x[3]);
    }
    return __ballot(any != 0) != 0;
}

// Sets the NaN codes of `bytes` bytes of LDS to 0.
__device__ inline void clear_nans(uint8_t* p, int bytes, int lane)
{
    for (int i = 16 * lane; i < bytes; i += 1024) {
        i32x4 x = *reinterpret_cast<const i32x4*>(p + i);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            x[j] &= (int)~((nan_bytes(x[j]) >> 7) * 255u);
        *reinterpret_cast<i32x4*>(p + i) = x;
    }
}

// An operand of E4M3 ones where `av` has NaN codes.
__device__ inline i32x8 nan_ones(const i32x8& av)
{
    i32x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = (int)((nan_bytes(av[i]) >> 7) * 0x38u);
    return x;
}

// Four E4M3 ones, the first `count` (at most 4) of them.
__device__ inline int ones(int count)
{
    return (int)(0x38383838u & (uint32_t)((1ull << (8 * min(max(count, 0), 4))) - 1));
}

// Largest of scores; NaN if one is NaN (an instruction for two values; fmax would
// first have to quieten each score).
__device__ inline float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A lane's part of a query row: f for which all |x| of the row on a score factor c are below
// 2^22 if c f <= 1 for its lanes (|code| <= 448).  Beyond, a score's FP32 product and the
// exact one may differ by more than the codes have room for (448 / 2^8).
template <int N>
__device__ inline float far_factor(const bf16x8* q, int d)
{
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    u16x8 m = {};
#pragma unroll
    for (int i = 0; i < N; ++i)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x8, q[i]) & (u16x8)((uint16_t)0x7FFF));
    uint16_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        top = m[i] > top ? m[i] : top;
    return __uint_as_float((uint32_t)top << 16) * (448.f / 0x1p22f * (float)d);
}

// ---- host side ----

// Workgroups of a launch, or hipErrorNotSupported: the threads of one are a 32-bit number.
// (128 bits: products of the caller's sizes)
inline hipError_t grid_of(__int128 workgroups, int threads, unsigned& grid)
{
    const bool fits = workgroups * threads < (__int128)1 << 32;
    grid = fits ? (unsigned)workgroups : 0;
    return fits ? hipSuccess : hipErrorNotSupported;
}

struct FwdParams {
    Batch bt;
    Cache cache;
    Heads q;
    void* out;
    float* lse;             // nullable
    float* ws;              // partial results of split tiles
    int out_bf16, Hq;
    Group gr;               // G = Hq / Hkv
    int causal, max_len;
    float c;                // log2(e) sm_scale q_descale
    int tiles, chunk, ranges;   // row tiles per (sequence, KV head); visits per range; most ranges
};

struct WeightParams {
    Batch bt;
    Cache cache;
    Heads q;
    const float* lse;
    float* w;
    int64_t sb, sh;
    int Hq;
    Group gr;
    int causal, max_len;
    float c;
};

struct EvictParams {
    Batch bt;
    Cache from, to;
    const int32_t* new_pages;   // [B][nb]
    const float* w;
    int64_t sb, sh;
    int budget, n_sink, n_recent, nb;
    int32_t* kept;
    int32_t* new_lens;
    float* new_w;               // nullable
};

// How a call of the attention is cut (host code; see cache_fwd.hip).
struct FwdPlan {
    int rows;               // query rows per tile
    int tiles;              // tiles per (sequence, KV head)
    int chunk, ranges;      // visits per range, ranges per tile (1: no split)
    size_t bytes;           // workspace
};
FwdPlan cache_fwd_plan(int B, int Hkv, int G, int max_q, int max_len, int d, int n_cu);

// Whether a call can be launched at all, by the fewest workgroups of a plan; the grids of
// one plan's launches (hipErrorNotSupported: too large).
bool cache_fwd_fits(int B, int Hkv, int G, int max_q);
struct FwdGrids {
    unsigned tiles, merges;
    int merge_rows;         // rows of a merging workgroup
};
hipError_t cache_fwd_grids(int B, int Hkv, int G, int max_q, int d, const FwdPlan& plan, FwdGrids& g);

hipError_t launch_rope(const Heads& x, const Heads& out, int T, int H, int d, int type, const Rotation& r, hipStream_t s);
hipError_t launch_append(const Batch& bt, const Cache& c, int d, int page, const Heads& k, const Heads& v, int type,
                         const Rotation& r, const Heads& q, const Heads& q_out, int Hq, hipStream_t s);
// (the launches: hipErrorNotSupported if a grid is too large, before any of them)
hipError_t launch_cache_fwd(FwdParams p, const FwdPlan& plan, int d, int page, bool e4m3, hipStream_t s);
hipError_t launch_cache_weights(const WeightParams& p, int d, int page, bool e4m3, int n_cu, hipStream_t s);
hipError_t launch_cache_evict(const EvictParams& p, int d, int page, hipStream_t s);

}  // namespace attn
