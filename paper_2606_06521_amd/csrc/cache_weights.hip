// Attention weight that cached tokens receive: per key the sum over the query
// rows of exp2(x - lse).
//
// D = Q K^T on the bf16 MFMA with the keys as columns: lane (n, g) holds rows
// 4 g .. 4 g + 3 of a 16-row tile for key n, so the sum over rows stays in the
// lane until the last row, and a key is owned by one workgroup: no atomics, one
// order of sums.
//
// Up to 64 rows (decode) the kernel streams K: a workgroup takes a range of
// visits of 128 keys, each of its eight waves every eighth one; a visit's codes go
// from their LDS stage to registers at once, so that the wave's next visit is on
// its way while this one is computed with Q in registers (two waves on a SIMD: one
// hides the other's latencies); the sums wait in LDS for one update of the weights
// at the end.  What bounds it is the stream of K: 16 x 8 heads x 8192 keys x 4 rows,
// d = 128, 34 us, 4.3 TB/s, of which 8 to begin and end.  With more rows (chunks) a
// workgroup takes 128 keys, widens them to bf16 registers once (64 keys a wave) and runs over
// the rows 64 at a time, the next 64 on their way into the other of two LDS stages,
// each wave two 16-row tiles of them; what bounds that is the vector work of every
// (row, key), at three waves a SIMD (39 % busy): 2 x 8 heads x 8192 keys x 1024 rows,
// ragged, 42 us.  Where blocks of 128 keys do not fill the GPU they are of 32 keys, and
// the waves share out the rows instead.
#include "cache_common.hpp"

#include <algorithm>
#include <type_traits>

namespace attn {

namespace {

constexpr int kStreamChunk = 32;     // visits of a range
constexpr int kStreamRows = 64;      // rows up to which K is streamed

// Row R of a (sequence, KV head): its lse in units of log2 (none: +inf, whose
// weights are 0) and the last key it sees (rows past the last: none).
__device__ inline void row_of(const WeightParams& p, const Seq& s, int hk, int R, int rows, float& lse2, int& last)
{
    const int at = min(R, rows - 1), i = p.gr.token(at);
    const float x = p.lse[(int64_t)(s.first + i) * p.Hq + hk * p.gr.G + (at - i * p.gr.G)];
    lse2 = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
    last = R >= rows ? -1 : last_key(s.pos0 + i, p.causal, s.len);
}

// Q operand of row R (past the last: any row): k-step 2 i + e of lane group g:
// channels 64 i + 16 g + 8 e on.
template <int KP, bool E4M3>
__device__ inline void q_rows(const WeightParams& p, const Seq& s, int hk, int R, int rows, int g, bf16x8* qf)
{
    R = min(R, rows - 1);
    const int i = p.gr.token(R);
    const int64_t at = (int64_t)(s.first + i) * p.q.st + (int64_t)(hk * p.gr.G + (R - i * p.gr.G)) * p.q.sh;
#pragma unroll
    for (int j = 0; j < 2 * KP; ++j)
        qf[j] = load_q8<E4M3>(p.q.data, at + 64 * (j / 2) + 16 * g + 8 * (j % 2));
}

__device__ inline float over_groups(float x)
{
    x += __shfl_xor(x, 16, 64);
    return halves_sum(x);
}

// x[g]
__device__ inline float of_group(int g, const float* x)
{
    const float lo = g & 1 ? x[1] : x[0], hi = g & 1 ? x[3] : x[2];
    return g & 2 ? hi : lo;
}

// K stage: row r's chunk c at chunk c ^ swz(r): 16 rows in a row are read without bank conflicts.
template <int D>
__device__ inline int stage_swz(int r)
{
    return D == 128 ? r & 7 : (r >> 1) & 3;
}

template <int D, int PAGE, bool E4M3, int RT>
__global__ void __launch_bounds__(512, 1) weights_stream_kernel(WeightParams p, int chunk, int ranges)
{
    constexpr int NW = 8, PPV = kVisit / PAGE, KT = kVisit / 16, KP = D / 64, CPR = D / 16;
    constexpr int STAGE = kVisit * D, NI = STAGE / 1024, IPP = NI / PPV;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[NW * STAGE];
    __shared__ float acc_w[kStreamChunk * kVisit];
    __shared__ int pids[kStreamChunk * PPV];
    __shared__ uint8_t kbyte[kStreamChunk * PPV];

    const int range = (int)(blockIdx.x % ranges);
    const int rest = (int)(blockIdx.x / ranges);
    const int hk = rest % p.cache.Hkv, b = rest / p.cache.Hkv;
    const Seq s = uniform(sequence(p.bt, b, p.max_len));
    const int visits = (s.len + kVisit - 1) / kVisit;
    const int v0 = range * chunk, v1 = min(v0 + chunk, visits);
    if (v0 >= v1 || s.n <= 0)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int rows = s.n * p.gr.G;
    const int np = (v1 - v0) * PPV;
    if (tid < np)
        pids[tid] = page_of(p.bt, p.cache.n_pages, b, v0 * PPV + tid);
    __syncthreads();

    const int lr = lane / CPR, lc = lane % CPR;
    const int k_off = lr * D + 16 * (lc ^ stage_swz<D>(lr));
    uint8_t* const st = lds + w * STAGE;
    auto issue = [&](int v) __attribute__((always_inline)) {
#pragma unroll
        for (int sub = 0; sub < PPV; ++sub) {
            const int pid = v < v1 ? __builtin_amdgcn_readfirstlane(pids[(v - v0) * PPV + sub]) : -1;
            const int left = pid < 0 ? 0 : min(max(s.len - (v * kVisit + sub * PAGE), 0), PAGE) * D;
            const i32x4 kb = bytes_buffer(p.cache.k + ((size_t)(pid < 0 ? 0 : pid) * p.cache.Hkv + hk) * (PAGE * D), left);
#pragma unroll
            for (int j = 0; j < IPP; ++j)
                load_lds16(kb, k_off, 1024 * j, st + 1024 * (sub * IPP + j));
        }
    };
    issue(v0 + w);
    // (these loads are younger: they wait for the first visit too)
    if (tid < np)
        kbyte[tid] = pids[tid] < 0 ? 127 : p.cache.ks[(size_t)pids[tid] * p.cache.Hkv + hk];
    bf16x8 qf[RT][2 * KP];
    float lse2[RT][4];
    int last[RT][4];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        q_rows<KP, E4M3>(p, s, hk, 16 * t + n, rows, g, qf[t]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            row_of(p, s, hk, 16 * t + 4 * g + r, rows, lse2[t][r], last[t][r]);
    }
    // the weights themselves, for the update at the end (one wait instead of one per entry)
    float* const out = p.w + (int64_t)b * p.sb + (int64_t)hk * p.sh + v0 * kVisit;
    constexpr int OWN = kStreamChunk * kVisit / (64 * NW);
    const int n_out = min((v1 - v0) * kVisit, s.len - v0 * kVisit);
    float old[OWN];
#pragma unroll
    for (int j = 0; j < OWN; ++j)
        old[j] = tid + 64 * NW * j < n_out ? out[tid + 64 * NW * j] : 0.f;
    // (used here, so that their wait is here and not in the loop)
#pragma unroll
    for (int j = 0; j < OWN; ++j)
        asm volatile("" : "+v"(old[j]));
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int j = 0; j < 2 * KP; ++j) {
            i32x4 x = __builtin_bit_cast(i32x4, qf[t][j]);
            asm volatile("" : "+v"(x));
            qf[t][j] = __builtin_bit_cast(bf16x8, x);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
            asm volatile("" : "+v"(lse2[t][r]));
    }
    __syncthreads();

    for (int v = v0 + w; v < v1; v += NW) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        i32x4 raw[KT][KP];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < KP; ++i)
                raw[kt][i] = *reinterpret_cast<const i32x4*>(st + (16 * kt + n) * D + 16 * ((4 * i + g) ^ stage_swz<D>(n)));
        // (all in registers: the stage takes the next visit)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        issue(v + NW);
        float sum[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const float c = score_factor(p.c, kbyte[(v - v0) * PPV + 16 * kt / PAGE]);
            bf16x8 kf[2 * KP];
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                kf[2 * i] = widen((uint32_t)raw[kt][i][0], (uint32_t)raw[kt][i][1]);
                kf[2 * i + 1] = widen((uint32_t)raw[kt][i][2], (uint32_t)raw[kt][i][3]);
            }
            const int t = v * kVisit + 16 * kt + n;
            sum[kt] = 0.f;
#pragma unroll
            for (int q = 0; q < RT; ++q) {
                if (RT > 1 && 16 * q >= rows)
                    break;
                f32x4 acc = {};
#pragma unroll
                for (int j = 0; j < 2 * KP; ++j)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[q][j], kf[j], acc, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[r], c, -lse2[q][r]));
                    sum[kt] += t <= last[q][r] ? x : 0.f;
                }
            }
        }
        // lane (n, g) keeps key n of tiles g and 4 + g: keys lane and 64 + lane
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
            sum[kt] = over_groups(sum[kt]);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
            acc_w[(v - v0) * kVisit + 64 * hf + lane] = of_group(g, sum + 4 * hf);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
        const int i = tid + 64 * NW * j;
        if (i < n_out && pids[i / PAGE] >= 0)
            out[i] = old[j] + acc_w[i];
    }
}

template <int D, int PAGE, bool E4M3, int KEYS>
__global__ void __launch_bounds__(256, 2) weights_tall_kernel(WeightParams p, int blocks)
{
    constexpr int KT = KEYS == 32 ? 2 : 4;          // 16-key tiles of a wave
    constexpr int NK = KEYS / (16 * KT), NR = 4 / NK;   // the waves: NK runs of keys, NR of a segment's rows
    constexpr int KP = D / 64, CPR = D / 16, WROWS = KEYS / 4;   // rows of K that a wave loads
    constexpr int STAGE = KEYS * D, LPW = (STAGE / 4 + 1023) / 1024;
    constexpr int SEG = 64;                         // rows of a segment
    constexpr int QB = E4M3 ? 1 : 2, QROW = QB * D; // bytes of a query's element and row
    constexpr int QC = QROW / 16, QRPI = 1024 / QROW, QLPW = 16 * QROW / 1024;   // chunks of a row, rows per load, loads of 16 rows
    __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t qst[2][SEG * QROW];
    __shared__ __attribute__((aligned(16))) float lse_s[2][SEG];
    __shared__ __attribute__((aligned(16))) int last_s[2][SEG];
    __shared__ float part_w[NR][KEYS];
    const int v = (int)(blockIdx.x % blocks);       // (causal: the first keys have the most rows)
    const int rest = (int)(blockIdx.x / blocks);
    const int hk = rest % p.cache.Hkv, b = rest / p.cache.Hkv;
    const Seq s = uniform(sequence(p.bt, b, p.max_len));
    const int t0 = v * KEYS;
    if (t0 >= s.len || s.n <= 0)
        return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int kh = w % NK, rh = w / NK;
    const int rows = s.n * p.gr.G;
    const int segs = (rows + SEG - 1) / SEG;
    // (causal: the rows before the first that sees key t0 add nothing)
    const int first = p.causal ? min(max(t0 - s.pos0, 0), s.n) * p.gr.G / SEG : 0;

    // a wave loads 16 rows of a segment, row r's chunk c at chunk c ^ qswz(r)
    auto qswz = [](int r) __attribute__((always_inline)) { return QROW >= 128 ? r & 7 : (r >> 1) & 3; };
    // (address and head of the lane's rows; from segment to segment they move on by 64
    // rows without a division; rows past the last read row 0, their weights are 0)
    const uint8_t* const q0 = static_cast<const uint8_t*>(p.q.data) + ((int64_t)s.first * p.q.st + (int64_t)hk * p.gr.G * p.q.sh) * QB;
    const int step_i = p.gr.token(SEG), step_h = SEG - step_i * p.gr.G;
    const int64_t step = (step_i * p.q.st + step_h * p.q.sh) * QB, carry = (p.q.st - p.gr.G * p.q.sh) * QB;
    int64_t q_at[QLPW];
    int q_head[QLPW];
#pragma unroll
    for (int j = 0; j < QLPW; ++j) {
        const int r = 16 * w + QRPI * j + lane / QC, R = SEG * first + r, i = p.gr.token(R);
        q_head[j] = R - i * p.gr.G;
        q_at[j] = (i * p.q.st + q_head[j] * p.q.sh) * QB + 16 * ((lane % QC) ^ qswz(r));
    }
    auto issue_q = [&](int seg, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < QLPW; ++j) {
            const bool in = SEG * seg + 16 * w + QRPI * j + lane / QC < rows;
            load_lds16(q0 + (in ? q_at[j] : 0), qst[buf] + 16 * w * QROW + 1024 * j);
            q_at[j] += step;
            q_head[j] += step_h;
            if (q_head[j] >= p.gr.G) {
                q_head[j] -= p.gr.G;
                q_at[j] += carry;
            }
        }
    };
    if (first < segs)
        issue_q(first, 0);
    // and WROWS rows of K, of one page
    const int lr = lane / CPR, lc = lane % CPR;
    const int k0 = t0 + WROWS * w;
    const int lpid = __builtin_amdgcn_readfirstlane(page_of(p.bt, p.cache.n_pages, b, k0 / PAGE));
    {
        const int left = lpid < 0 ? 0 : min(min(max(s.len - k0, 0), WROWS), PAGE - k0 % PAGE) * D;
        const i32x4 kb = bytes_buffer(p.cache.k + ((size_t)(lpid < 0 ? 0 : lpid) * p.cache.Hkv + hk) * (PAGE * D) + k0 % PAGE * D, left);
        // (fewer rows than a load holds: the other lanes stay out)
        if (lr < WROWS) {
#pragma unroll
            for (int j = 0; j < LPW; ++j)
                load_lds16(kb, lr * D + 16 * (lc ^ stage_swz<D>(lr)), 1024 * j, lds + w * (WROWS * D) + 1024 * j);
        }
    }
    const int pid = __builtin_amdgcn_readfirstlane(page_of(p.bt, p.cache.n_pages, b, (t0 + 16 * KT * kh) / PAGE));
    const float c = pid < 0 ? 0.f : score_factor(p.c, p.cache.ks[(size_t)pid * p.cache.Hkv + hk]);
    float lse2 = 0.f;
    int last = -1;
    if (tid < SEG) {
        row_of(p, s, hk, SEG * first + tid, rows, lse2, last);
        lse_s[0][tid] = lse2;
        last_s[0][tid] = last;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    bf16x8 kf[KT][2 * KP];
    float sum[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const int r = 16 * KT * kh + 16 * kt + n;
        sum[kt] = 0.f;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const i32x4 x = *reinterpret_cast<const i32x4*>(lds + r * D + 16 * ((4 * i + g) ^ stage_swz<D>(r)));
            kf[kt][2 * i] = widen((uint32_t)x[0], (uint32_t)x[1]);
            kf[kt][2 * i + 1] = widen((uint32_t)x[2], (uint32_t)x[3]);
        }
    }
    int buf = 0;
    for (int seg = first; seg < segs; ++seg, buf ^= 1) {
        if (seg + 1 < segs) {
            if (tid < SEG)
                row_of(p, s, hk, SEG * (seg + 1) + tid, rows, lse2, last);
            issue_q(seg + 1, buf ^ 1);
        }
        // every row of the segment sees every key of the block
        const bool all = SEG * (seg + 1) <= rows && s.pos0 + p.gr.token(SEG * seg) >= (p.causal ? t0 + KEYS - 1 : 0) && t0 + KEYS <= s.len;
        auto tiles = [&](auto masked) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < NK; ++q) {
                const int r0 = 16 * (NK * rh + q);
                bf16x8 qf[2 * KP];
#pragma unroll
                for (int i = 0; i < KP; ++i) {
                    const uint8_t* const at = qst[buf] + (r0 + n) * QROW;
                    if constexpr (E4M3) {
                        const i32x4 x = *reinterpret_cast<const i32x4*>(at + 16 * ((4 * i + g) ^ qswz(n)));
                        qf[2 * i] = widen((uint32_t)x[0], (uint32_t)x[1]);
                        qf[2 * i + 1] = widen((uint32_t)x[2], (uint32_t)x[3]);
                    } else {
                        qf[2 * i] = *reinterpret_cast<const bf16x8*>(at + 16 * ((8 * i + 2 * g) ^ qswz(n)));
                        qf[2 * i + 1] = *reinterpret_cast<const bf16x8*>(at + 16 * ((8 * i + 2 * g + 1) ^ qswz(n)));
                    }
                }
                const f32x4 l4 = *reinterpret_cast<const f32x4*>(&lse_s[buf][r0 + 4 * g]);
                const i32x4 e4 = *reinterpret_cast<const i32x4*>(&last_s[buf][r0 + 4 * g]);
                // (the tiles' chains of matrix instructions side by side: none waits for itself)
                f32x4 acc[KT];
#pragma unroll
                for (int j = 0; j < 2 * KP; ++j)
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
                        acc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[j], kf[kt][j], j == 0 ? f32x4{} : acc[kt], 0, 0, 0);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const int t = t0 + 16 * (KT * kh + kt) + n;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[kt][r], c, -l4[r]));
                        sum[kt] += !decltype(masked)::value || t <= e4[r] ? x : 0.f;
                    }
                }
            }
        };
        if (all)
            tiles(std::false_type{});
        else
            tiles(std::true_type{});
        // the next segment is there, and everyone is done with this one
        if (tid < SEG) {
            lse_s[buf ^ 1][tid] = lse2;
            last_s[buf ^ 1][tid] = last;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
        sum[kt] = over_groups(sum[kt]);
    // lane (n, g) has key n of tile g
    const float x = KT == 4 ? of_group(g, sum) : g & 1 ? sum[1] : sum[0];
    const int at = 16 * KT * kh + lane % (16 * KT);
    if (lane < 16 * KT)
        part_w[rh][at] = x;
    __syncthreads();
    const int t = t0 + at;
    if (rh == 0 && lane < 16 * KT && t < s.len && pid >= 0) {
        float total = part_w[0][at];
#pragma unroll
        for (int i = 1; i < NR; ++i)
            total += part_w[i][at];
        p.w[(int64_t)b * p.sb + (int64_t)hk * p.sh + t] += total;
    }
}

}  // namespace

hipError_t launch_cache_weights(const WeightParams& p, int d, int page, bool e4m3, int n_cu, hipStream_t s)
{
    const int visits = (p.max_len + kVisit - 1) / kVisit;
    const int64_t heads = (int64_t)p.bt.B * p.cache.Hkv, rows = (int64_t)p.bt.max_q * p.gr.G;
    const bool tall = rows > kStreamRows;
    // ranges that fill the GPU, of at least a visit per wave
    const int64_t want = std::max<int64_t>(1, n_cu / heads);
    const int chunk = (int)std::min<int64_t>(std::max<int64_t>(8, (visits + want - 1) / want), kStreamChunk);
    const int ranges = (visits + chunk - 1) / chunk;
    // Keys of a block with many rows: 128, or 32 where that leaves CUs without a block (1 x 2
    // heads x 2048 keys, 256 x 4 rows: 19.6 us with 128, 13.2 with 32; 1 x 8 x 5269, 607 x 8 rows,
    // 336 blocks: 82 and 83; 8 x 8 x 1024, 64 x 4 rows, 512 blocks: 12 and 16)
    const int keys = heads * visits < n_cu ? 32 : 128;
    const int blocks = (p.max_len + keys - 1) / keys;
    unsigned grid;
    const hipError_t e = grid_of((__int128)heads * (tall ? blocks : ranges), tall ? 256 : 512, grid);
    if (e != hipSuccess)
        return e;
    auto by_type = [&](auto dc, auto pc, auto ec) {
        constexpr int D = decltype(dc)::value, PAGE = decltype(pc)::value;
        constexpr bool E = decltype(ec)::value;
        auto tall_of = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, p, blocks); };
        if (tall && keys == 128)
            tall_of(weights_tall_kernel<D, PAGE, E, 128>);
        else if (tall)
            tall_of(weights_tall_kernel<D, PAGE, E, 32>);
        else if (rows <= 16)
            hipLaunchKernelGGL((weights_stream_kernel<D, PAGE, E, 1>), dim3(grid), dim3(512), 0, s, p, chunk, ranges);
        else
            hipLaunchKernelGGL((weights_stream_kernel<D, PAGE, E, kStreamRows / 16>), dim3(grid), dim3(512), 0, s, p, chunk,
                               ranges);
        return hipGetLastError();
    };
    using std::integral_constant;
    auto by_size = [&](auto ec) {
        if (d == 64)
            return page == 64 ? by_type(integral_constant<int, 64>{}, integral_constant<int, 64>{}, ec)
                              : by_type(integral_constant<int, 64>{}, integral_constant<int, 128>{}, ec);
        return page == 64 ? by_type(integral_constant<int, 128>{}, integral_constant<int, 64>{}, ec)
                          : by_type(integral_constant<int, 128>{}, integral_constant<int, 128>{}, ec);
    };
    return e4m3 ? by_size(std::true_type{}) : by_size(std::false_type{});
}

}  // namespace attn
