// C ABI of the KV cache (declared in include/attn_fp8_cache.h and attn_fp8_parts.h): argument
// validation and launch on the caller's stream.  No state is kept and no memory
// is allocated.
#include "../../include/attn_fp8_cache.h"
#include "../../include/attn_fp8_parts.h"
#include "cache_common.hpp"

#include <math.h>

namespace {

using attn::Batch;
using attn::Cache;
using attn::Heads;

bool misaligned(const void* p, uintptr_t a) { return (uintptr_t)p % a != 0; }

int type_size(int type)
{
    switch (type) {
    case ATTN_TYPE_F32:
        return 4;
    case ATTN_TYPE_BF16:
    case ATTN_TYPE_F16:
        return 2;
    case ATTN_TYPE_E4M3:
        return 1;
    default:
        return 0;
    }
}

bool is_input_type(int type) { return type == ATTN_TYPE_F32 || type == ATTN_TYPE_BF16 || type == ATTN_TYPE_F16; }

// Sizes of a cache and a batch (no pointer is looked at).
int check_sizes(const attn_fp8_cache* c, const attn_fp8_batch* bt)
{
    if (!c || !bt || c->n_pages < 0 || c->Hkv < 1 || c->page < 1 || c->d < 1 || bt->B < 0 || bt->W < 0 || bt->T < 0 ||
        bt->max_q < 1)
        return ATTN_ERR_INVALID_ARG;
    if (c->d != 64 && c->d != 128)
        return ATTN_ERR_UNSUPPORTED;
    if (c->page != 64 && c->page != 128)
        return ATTN_ERR_UNSUPPORTED;
    // (the merge of a split call holds at most 4096 ranges; the distance of a key and a
    // token's position fits 32 bits)
    if ((int64_t)bt->W * c->page > 1 << 26 || c->Hkv > 1 << 16 || bt->max_q > 1 << 26 || bt->T > 1 << 30)
        return ATTN_ERR_UNSUPPORTED;
    return ATTN_OK;
}

int check_cache(const attn_fp8_cache* c)
{
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || misaligned(c->k, 16) || misaligned(c->v, 16))
        return ATTN_ERR_INVALID_ARG;
    return ATTN_OK;
}

int check_batch(const attn_fp8_batch* bt, bool with_tokens)
{
    if ((!bt->pages && bt->W > 0) || !bt->lens || misaligned(bt->pages, 4) || misaligned(bt->lens, 4) || misaligned(bt->cu, 4))
        return ATTN_ERR_INVALID_ARG;
    if (with_tokens && !bt->cu && (bt->T % bt->B != 0 || bt->T / bt->B > bt->max_q))
        return ATTN_ERR_INVALID_ARG;
    return ATTN_OK;
}

int check_heads(const attn_fp8_heads* h)
{
    const int size = type_size(h->type);
    if (!size || !h->data || misaligned(h->data, 16) || h->stride_t < 0 || h->stride_h < 0 || h->stride_t * size % 16 != 0 ||
        h->stride_h * size % 16 != 0)
        return ATTN_ERR_INVALID_ARG;
    return ATTN_OK;
}

int check_rotation(const attn_fp8_rotation* r, int d)
{
    if (!r->table || misaligned(r->table, 16) || misaligned(r->positions, 4) || r->n_pos < 1 || r->rot < 1 || r->rot > d ||
        (r->layout != ATTN_ROPE_HALF && r->layout != ATTN_ROPE_INTERLEAVED))
        return ATTN_ERR_INVALID_ARG;
    return r->rot % 16 == 0 ? ATTN_OK : ATTN_ERR_UNSUPPORTED;
}

Cache cache_of(const attn_fp8_cache* c)
{
    return {static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, c->n_pages, c->Hkv};
}

Batch batch_of(const attn_fp8_batch* bt)
{
    return {bt->pages, bt->lens, bt->cu, bt->B, bt->W, bt->T, bt->max_q, bt->cu || !bt->B ? 0 : bt->T / bt->B};
}

Heads heads_of(const attn_fp8_heads* h) { return {h->data, h->stride_t, h->stride_h}; }

attn::Rotation rotation_of(const attn_fp8_rotation* r)
{
    return {r->table, r->positions, r->n_pos, r->rot, r->layout};
}

// (a launch that would need too large a grid was not tried)
int status(hipError_t e) { return e == hipSuccess ? ATTN_OK : e == hipErrorNotSupported ? ATTN_ERR_UNSUPPORTED : ATTN_ERR_HIP; }

// Elements of four bytes; none at a null address.
struct Span {
    const void* at;
    __int128 n;         // (strides are the caller's: any number of 64 bits)
};

bool overlap(const Span& x, const Span& y)
{
    const __int128 a = (uintptr_t)x.at, b = (uintptr_t)y.at;
    return a && b && x.n > 0 && y.n > 0 && a < b + 4 * y.n && b < a + 4 * x.n;
}

// What a raw score is multiplied by on a block scale of 1.
float factor_of(float sm_scale, float q_descale) { return (float)(1.4426950408889634074 * (double)sm_scale * (double)q_descale); }

// The sizes and scalars that attention and weights share.
int check_attention(const attn_fp8_cache* c, const attn_fp8_batch* bt, int Hq, int causal, float sm_scale, float q_descale,
                    int max_len)
{
    const int st = check_sizes(c, bt);
    if (st != ATTN_OK)
        return st;
    if (Hq < 1 || Hq % c->Hkv != 0 || max_len < 0 || (causal != 0 && causal != 1) || !(sm_scale > 0.f) || !isfinite(sm_scale) ||
        !(q_descale > 0.f) || !isfinite(q_descale) || !isnormal(factor_of(sm_scale, q_descale)))
        return ATTN_ERR_INVALID_ARG;
    // (the row numbers of a sequence and KV head times the group stay below 2^32)
    const int G = Hq / c->Hkv;
    unsigned heads;
    if (G > 256 || (int64_t)G * bt->max_q > 1 << 24 || attn::grid_of((__int128)bt->B * c->Hkv, 256, heads) != hipSuccess)
        return ATTN_ERR_UNSUPPORTED;
    return ATTN_OK;
}

int longest(const attn_fp8_cache* c, const attn_fp8_batch* bt, int max_len)
{
    const int most = bt->W * c->page;
    return max_len > 0 && max_len < most ? max_len : most;
}

int device_cus(int& n_cu)
{
    int dev = 0;
    n_cu = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
        return ATTN_ERR_HIP;
    return ATTN_OK;
}

// What the attention calls share: pointers, types and the launch parameters.
int check_fwd(const attn_fp8_cache* cache, const attn_fp8_batch* batch, const attn_fp8_heads* q, const void* out,
              const float* lse, const void* workspace)
{
    int st;
    if ((st = check_cache(cache)) != ATTN_OK || (st = check_batch(batch, true)) != ATTN_OK || (st = check_heads(q)) != ATTN_OK)
        return st;
    if ((q->type != ATTN_TYPE_BF16 && q->type != ATTN_TYPE_E4M3) || !out || misaligned(out, 16) || misaligned(lse, 4) ||
        misaligned(workspace, 256))
        return ATTN_ERR_INVALID_ARG;
    return ATTN_OK;
}

void fill_fwd(attn::FwdParams& p, const attn_fp8_cache* cache, const attn_fp8_batch* batch, const attn_fp8_heads* q, int Hq,
              void* out, int out_type, float* lse, int causal, float sm_scale, float q_descale, int max_len, void* workspace)
{
    p.bt = batch_of(batch);
    p.cache = cache_of(cache);
    p.q = heads_of(q);
    p.out = out;
    p.lse = lse;
    p.ws = static_cast<float*>(workspace);
    p.out_bf16 = out_type == ATTN_TYPE_BF16;
    p.Hq = Hq;
    p.gr = attn::group_of(Hq / cache->Hkv);
    p.causal = causal;
    p.max_len = longest(cache, batch, max_len);
    p.c = factor_of(sm_scale, q_descale);
}

// Lists of `take` blocks for runs of new tokens: how many a KV head has.
int check_lists(const attn_fp8_cache* c, const attn_fp8_batch* bt, int take, int most, int run, int64_t& runs)
{
    if (take < 1 || run < 1)
        return ATTN_ERR_INVALID_ARG;
    runs = ((int64_t)bt->max_q + run - 1) / run;
    unsigned lists;
    if (take > most || attn::grid_of((__int128)bt->B * c->Hkv * runs, 256, lists) != hipSuccess)
        return ATTN_ERR_UNSUPPORTED;
    return ATTN_OK;
}

// The plan of an attention over lists; ATTN_ERR_UNSUPPORTED if it cannot be launched.
int plan_blocks(const attn_fp8_cache* c, const attn_fp8_batch* bt, int Hq, int take, int run, int64_t runs, attn::FwdPlan& pl)
{
    const int G = Hq / c->Hkv;
    const int64_t lists = (int64_t)bt->B * c->Hkv * runs;
    run = run < bt->max_q ? run : bt->max_q;
    unsigned fewest;
    if (attn::grid_of((__int128)lists * (((int64_t)run * G + 127) / 128), 256, fewest) != hipSuccess)
        return ATTN_ERR_UNSUPPORTED;
    int n_cu = 0;
    if (device_cus(n_cu) != ATTN_OK)
        return ATTN_ERR_HIP;
    pl = attn::blocks_plan(lists, G, run, take, c->page, c->d, n_cu);
    attn::FwdGrids g;
    return attn::blocks_grids(lists, (int64_t)run * G, c->d, pl, g) == hipSuccess ? ATTN_OK : ATTN_ERR_UNSUPPORTED;
}

int plan_shared(const attn_fp8_cache* c, const attn_fp8_batch* bt, int shared, int Hq, int max_len, attn::SharedPlan& pl)
{
    const int G = Hq / c->Hkv;
    if (shared < 0 || shared > bt->W)
        return ATTN_ERR_INVALID_ARG;
    if ((int64_t)G * bt->T > 1 << 24 || !attn::cache_fwd_fits(bt->B, c->Hkv, G, bt->max_q))
        return ATTN_ERR_UNSUPPORTED;
    if (bt->B == 0 || bt->T == 0)
        return ATTN_OK;
    int n_cu = 0;
    if (device_cus(n_cu) != ATTN_OK)
        return ATTN_ERR_HIP;
    pl = attn::shared_plan(bt->B, c->Hkv, G, bt->T, bt->max_q, shared, longest(c, bt, max_len), c->page, c->d, n_cu);
    attn::SharedGrids g;
    return attn::shared_grids(bt->B, c->Hkv, G, bt->max_q, c->d, pl, g) == hipSuccess ? ATTN_OK : ATTN_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

int attn_fp8_rope(const attn_fp8_heads* x, const attn_fp8_heads* out, int T, int H, int d, const attn_fp8_rotation* rotation,
                  void* stream)
{
    if (!x || !out || !rotation || T < 0 || H < 0 || d < 1)
        return ATTN_ERR_INVALID_ARG;
    if (d % 16 != 0 || d > 1024)
        return ATTN_ERR_UNSUPPORTED;
    if (T == 0 || H == 0)
        return ATTN_OK;
    int st = check_heads(x);
    if (st == ATTN_OK)
        st = check_heads(out);
    if (st != ATTN_OK)
        return st;
    if (!is_input_type(x->type) || x->type != out->type || !rotation->positions)
        return ATTN_ERR_INVALID_ARG;
    if ((st = check_rotation(rotation, d)) != ATTN_OK)
        return st;
    return status(attn::launch_rope(heads_of(x), heads_of(out), T, H, d, x->type, rotation_of(rotation),
                                    static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_append(const attn_fp8_cache* cache, const attn_fp8_batch* batch, const attn_fp8_heads* k,
                          const attn_fp8_heads* v, const attn_fp8_rotation* rotation, const attn_fp8_heads* q,
                          const attn_fp8_heads* q_out, int Hq, void* stream)
{
    int st = check_sizes(cache, batch);
    if (st != ATTN_OK)
        return st;
    if (!k || !v || !q != !q_out || (q && (!rotation || Hq < 1)))
        return ATTN_ERR_INVALID_ARG;
    if (batch->B == 0 || batch->T == 0)
        return ATTN_OK;
    if ((st = check_cache(cache)) != ATTN_OK || (st = check_batch(batch, true)) != ATTN_OK || (st = check_heads(k)) != ATTN_OK ||
        (st = check_heads(v)) != ATTN_OK)
        return st;
    if (!is_input_type(k->type) || v->type != k->type)
        return ATTN_ERR_INVALID_ARG;
    if (rotation && (st = check_rotation(rotation, cache->d)) != ATTN_OK)
        return st;
    if (q) {
        if ((st = check_heads(q)) != ATTN_OK || (st = check_heads(q_out)) != ATTN_OK)
            return st;
        if (q->type != k->type || q_out->type != k->type)
            return ATTN_ERR_INVALID_ARG;
    }
    return status(attn::launch_append(batch_of(batch), cache_of(cache), cache->d, cache->page, heads_of(k), heads_of(v), k->type,
                                      rotation ? rotation_of(rotation) : attn::Rotation{}, q ? heads_of(q) : Heads{},
                                      q ? heads_of(q_out) : Heads{}, Hq, static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_workspace_bytes(const attn_fp8_cache* cache, const attn_fp8_batch* batch, int Hq, int max_len, size_t* bytes)
{
    if (!bytes)
        return ATTN_ERR_INVALID_ARG;
    *bytes = 0;
    const int st = check_attention(cache, batch, Hq, 1, 1.f, 1.f, max_len);
    if (st != ATTN_OK || batch->B == 0 || batch->T == 0)
        return st;
    if (!attn::cache_fwd_fits(batch->B, cache->Hkv, Hq / cache->Hkv, batch->max_q))
        return ATTN_ERR_UNSUPPORTED;
    int n_cu = 0;
    if (device_cus(n_cu) != ATTN_OK)
        return ATTN_ERR_HIP;
    const int G = Hq / cache->Hkv;
    const attn::FwdPlan pl = attn::cache_fwd_plan(batch->B, cache->Hkv, G, batch->max_q, longest(cache, batch, max_len), cache->d, n_cu);
    attn::FwdGrids g;
    if (attn::cache_fwd_grids(batch->B, cache->Hkv, G, batch->max_q, cache->d, pl, g) != hipSuccess)
        return ATTN_ERR_UNSUPPORTED;
    *bytes = pl.bytes;
    return ATTN_OK;
}

int attn_fp8_cache_fwd(const attn_fp8_cache* cache, const attn_fp8_batch* batch, const attn_fp8_heads* q, int Hq, void* out,
                       int out_type, float* lse, int causal, float sm_scale, float q_descale, int max_len, void* workspace,
                       size_t workspace_bytes, void* stream)
{
    int st = check_attention(cache, batch, Hq, causal, sm_scale, q_descale, max_len);
    if (st != ATTN_OK)
        return st;
    if (!q || (out_type != ATTN_TYPE_BF16 && out_type != ATTN_TYPE_F32))
        return ATTN_ERR_INVALID_ARG;
    if (batch->B == 0 || batch->T == 0)
        return ATTN_OK;
    if ((st = check_fwd(cache, batch, q, out, lse, workspace)) != ATTN_OK)
        return st;
    if (!attn::cache_fwd_fits(batch->B, cache->Hkv, Hq / cache->Hkv, batch->max_q))
        return ATTN_ERR_UNSUPPORTED;
    int n_cu = 0;
    if ((st = device_cus(n_cu)) != ATTN_OK)
        return st;
    attn::FwdParams p{};
    fill_fwd(p, cache, batch, q, Hq, out, out_type, lse, causal, sm_scale, q_descale, max_len, workspace);
    const attn::FwdPlan pl = attn::cache_fwd_plan(batch->B, cache->Hkv, p.gr.G, batch->max_q, p.max_len, cache->d, n_cu);
    if (pl.bytes > 0 && (!workspace || workspace_bytes < pl.bytes))
        return ATTN_ERR_INVALID_ARG;
    return status(attn::launch_cache_fwd(p, pl, cache->d, cache->page, q->type == ATTN_TYPE_E4M3, static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_weights(const attn_fp8_cache* cache, const attn_fp8_batch* batch, const attn_fp8_heads* q, int Hq,
                           const float* lse, int causal, float sm_scale, float q_descale, int max_len, float* weights,
                           int64_t stride_b, int64_t stride_h, void* stream)
{
    int st = check_attention(cache, batch, Hq, causal, sm_scale, q_descale, max_len);
    if (st != ATTN_OK)
        return st;
    if (!q || stride_b < 0 || stride_h < 0)
        return ATTN_ERR_INVALID_ARG;
    const int most = longest(cache, batch, max_len);
    if (batch->B == 0 || batch->T == 0 || most == 0)
        return ATTN_OK;
    if ((st = check_cache(cache)) != ATTN_OK || (st = check_batch(batch, true)) != ATTN_OK || (st = check_heads(q)) != ATTN_OK)
        return st;
    if ((q->type != ATTN_TYPE_BF16 && q->type != ATTN_TYPE_E4M3) || !lse || !weights || misaligned(lse, 4) ||
        misaligned(weights, 4) || stride_h < most)
        return ATTN_ERR_INVALID_ARG;
    // (rows are updated without atomics: sequences outermost or heads outermost, none over another)
    const __int128 sb = stride_b, sh = stride_h;
    if (batch->B > 1 && sb < (cache->Hkv - 1) * sh + most && (sb < most || (cache->Hkv > 1 && sh < (batch->B - 1) * sb + most)))
        return ATTN_ERR_INVALID_ARG;
    attn::WeightParams p{};
    p.bt = batch_of(batch);
    p.cache = cache_of(cache);
    p.q = heads_of(q);
    p.lse = lse;
    p.w = weights;
    p.sb = stride_b;
    p.sh = stride_h;
    p.Hq = Hq;
    p.gr = attn::group_of(Hq / cache->Hkv);
    p.causal = causal;
    p.max_len = most;
    p.c = factor_of(sm_scale, q_descale);
    int n_cu = 0;
    if ((st = device_cus(n_cu)) != ATTN_OK)
        return st;
    return status(attn::launch_cache_weights(p, cache->d, cache->page, q->type == ATTN_TYPE_E4M3, n_cu, static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_evict(const attn_fp8_cache* from, const attn_fp8_batch* batch, const attn_fp8_cache* to,
                         const int32_t* new_pages, const float* weights, int64_t stride_b, int64_t stride_h, int budget,
                         int n_sink, int n_recent, int32_t* kept, int32_t* new_lens, float* new_weights, void* stream)
{
    int st = check_sizes(from, batch);
    if (st == ATTN_OK)
        st = check_sizes(to, batch);
    if (st != ATTN_OK)
        return st;
    if (to->Hkv != from->Hkv || to->page != from->page || to->d != from->d || stride_b < 0 || stride_h < 0 || budget < 1 ||
        n_sink < 0 || n_recent < 0 || (batch->B > 0 && from->n_pages < 1))
        return ATTN_ERR_INVALID_ARG;    // (rows without a page load those of page 0)
    if (budget > 1 << 20)
        return ATTN_ERR_UNSUPPORTED;
    if (batch->B == 0)
        return ATTN_OK;
    if ((st = check_cache(from)) != ATTN_OK || (st = check_cache(to)) != ATTN_OK || (st = check_batch(batch, false)) != ATTN_OK)
        return st;
    if (!new_pages || !weights || !kept || !new_lens || misaligned(new_pages, 4) || misaligned(weights, 4) || misaligned(kept, 4) ||
        misaligned(new_lens, 4) || misaligned(new_weights, 4) || stride_h < (int64_t)batch->W * from->page)
        return ATTN_ERR_INVALID_ARG;
    // (workgroups read lens, pages and weights while others write; rows of weights end at W * page)
    const int64_t heads = (int64_t)batch->B * from->Hkv, nb = (budget + from->page - 1) / from->page;
    const Span outs[] = {{kept, (__int128)heads * budget}, {new_lens, batch->B}, {new_weights, (__int128)heads * budget}};
    const Span ins[] = {{batch->lens, batch->B},
                        {batch->pages, (int64_t)batch->B * batch->W},
                        {new_pages, batch->B * nb},
                        {weights, (__int128)(batch->B - 1) * stride_b + (__int128)(from->Hkv - 1) * stride_h +
                                      (int64_t)batch->W * from->page}};
    for (int i = 0; i < 3; ++i) {
        for (const Span& in : ins)
            if (overlap(outs[i], in))
                return ATTN_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlap(outs[i], outs[j]))
                return ATTN_ERR_INVALID_ARG;
    }
    attn::EvictParams p{};
    p.bt = batch_of(batch);
    p.from = cache_of(from);
    p.to = cache_of(to);
    p.new_pages = new_pages;
    p.w = weights;
    p.sb = stride_b;
    p.sh = stride_h;
    p.budget = budget;
    p.n_sink = n_sink;
    p.n_recent = n_recent;
    p.nb = (int)nb;
    p.kept = kept;
    p.new_lens = new_lens;
    p.new_w = new_weights;
    return status(attn::launch_cache_evict(p, from->d, from->page, static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_bounds(const attn_fp8_cache* cache, const attn_fp8_batch* batch, void* bounds, void* stream)
{
    int st = check_sizes(cache, batch);
    if (st != ATTN_OK || batch->B == 0)
        return st;
    if ((st = check_cache(cache)) != ATTN_OK || (st = check_batch(batch, true)) != ATTN_OK)
        return st;
    if (!bounds || misaligned(bounds, 16))
        return ATTN_ERR_INVALID_ARG;
    if (batch->T == 0 || batch->W == 0)
        return ATTN_OK;
    attn::BoundsParams p{};
    p.bt = batch_of(batch);
    p.cache = cache_of(cache);
    p.bounds = static_cast<uint8_t*>(bounds);
    // (n tokens lie in at most this many pages)
    const int most = (batch->max_q + cache->page - 2) / cache->page + 1;
    return status(attn::launch_cache_bounds(p, most < batch->W ? most : batch->W, cache->d, cache->page, static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_select(const attn_fp8_cache* cache, const attn_fp8_batch* batch, const attn_fp8_heads* q, int Hq,
                          const void* bounds, int32_t* blocks, int take, int run, int n_first, int n_last, int causal,
                          int max_len, void* workspace, size_t workspace_bytes, void* stream)
{
    int64_t runs;
    int st = check_attention(cache, batch, Hq, causal, 1.f, 1.f, max_len);
    if (st == ATTN_OK)
        st = check_lists(cache, batch, take, attn::kMaxChoice, run, runs);
    if (st != ATTN_OK)
        return st;
    if (!q || n_first < 0 || n_last < 0 || (int64_t)n_first + n_last > take)
        return ATTN_ERR_INVALID_ARG;
    const int most = longest(cache, batch, max_len);
    if (most > attn::kMaxChoice * cache->page)
        return ATTN_ERR_UNSUPPORTED;
    if (batch->B == 0)
        return ATTN_OK;
    if ((st = check_cache(cache)) != ATTN_OK || (st = check_batch(batch, true)) != ATTN_OK ||
        (batch->T > 0 && (st = check_heads(q)) != ATTN_OK))
        return st;
    if ((q->type != ATTN_TYPE_BF16 && q->type != ATTN_TYPE_E4M3) || !bounds || misaligned(bounds, 16) || !blocks || misaligned(blocks, 4) ||
        misaligned(workspace, 256))
        return ATTN_ERR_INVALID_ARG;
    const attn::SelectPlan pl = attn::select_plan((int64_t)batch->B * cache->Hkv * runs, (most + cache->page - 1) / cache->page);
    if (pl.bytes > 0 && (!workspace || workspace_bytes < pl.bytes))
        return ATTN_ERR_INVALID_ARG;
    attn::SelectParams p{};
    p.bt = batch_of(batch);
    p.cache = cache_of(cache);
    p.q = heads_of(q);
    p.bounds = static_cast<const uint8_t*>(bounds);
    p.blocks = blocks;
    p.take = take;
    p.run = run < batch->max_q ? run : batch->max_q;
    p.runs = (int)runs;
    p.n_first = n_first;
    p.n_last = n_last;
    p.gr = attn::group_of(Hq / cache->Hkv);
    p.causal = causal;
    p.max_len = most;
    p.keys = static_cast<uint32_t*>(workspace);
    return status(attn::launch_cache_select(p, pl, cache->d, cache->page, q->type == ATTN_TYPE_E4M3, static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_select_workspace_bytes(const attn_fp8_cache* cache, const attn_fp8_batch* batch, int Hq, int take, int run,
                                          int max_len, size_t* bytes)
{
    if (!bytes)
        return ATTN_ERR_INVALID_ARG;
    *bytes = 0;
    int64_t runs;
    int st = check_attention(cache, batch, Hq, 1, 1.f, 1.f, max_len);
    if (st == ATTN_OK)
        st = check_lists(cache, batch, take, attn::kMaxChoice, run, runs);
    if (st != ATTN_OK)
        return st;
    const int most = longest(cache, batch, max_len);
    if (most > attn::kMaxChoice * cache->page)
        return ATTN_ERR_UNSUPPORTED;
    if (batch->B == 0)
        return ATTN_OK;
    *bytes = attn::select_plan((int64_t)batch->B * cache->Hkv * runs, (most + cache->page - 1) / cache->page).bytes;
    return ATTN_OK;
}

int attn_fp8_cache_blocks_workspace_bytes(const attn_fp8_cache* cache, const attn_fp8_batch* batch, int Hq, int take, int run,
                                          size_t* bytes)
{
    if (!bytes)
        return ATTN_ERR_INVALID_ARG;
    *bytes = 0;
    int64_t runs;
    int st = check_attention(cache, batch, Hq, 1, 1.f, 1.f, 0);
    if (st == ATTN_OK)
        st = check_lists(cache, batch, take, 1 << 19, run, runs);
    if (st != ATTN_OK || batch->B == 0 || batch->T == 0)
        return st;
    attn::FwdPlan pl;
    st = plan_blocks(cache, batch, Hq, take, run, runs, pl);
    if (st == ATTN_OK)
        *bytes = pl.bytes;
    return st;
}

int attn_fp8_cache_fwd_blocks(const attn_fp8_cache* cache, const attn_fp8_batch* batch, const attn_fp8_heads* q, int Hq,
                              const int32_t* blocks, int take, int run, void* out, int out_type, float* lse, int causal,
                              float sm_scale, float q_descale, void* workspace, size_t workspace_bytes, void* stream)
{
    int64_t runs;
    int st = check_attention(cache, batch, Hq, causal, sm_scale, q_descale, 0);
    if (st == ATTN_OK)
        st = check_lists(cache, batch, take, 1 << 19, run, runs);
    if (st != ATTN_OK)
        return st;
    if (!q || (out_type != ATTN_TYPE_BF16 && out_type != ATTN_TYPE_F32))
        return ATTN_ERR_INVALID_ARG;
    if (batch->B == 0 || batch->T == 0)
        return ATTN_OK;
    if ((st = check_fwd(cache, batch, q, out, lse, workspace)) != ATTN_OK)
        return st;
    if (!blocks || misaligned(blocks, 4))
        return ATTN_ERR_INVALID_ARG;
    attn::FwdPlan pl;
    if ((st = plan_blocks(cache, batch, Hq, take, run, runs, pl)) != ATTN_OK)
        return st;
    if (pl.bytes > 0 && (!workspace || workspace_bytes < pl.bytes))
        return ATTN_ERR_INVALID_ARG;
    attn::BlocksParams p{};
    fill_fwd(p, cache, batch, q, Hq, out, out_type, lse, causal, sm_scale, q_descale, 0, workspace);
    p.blocks = blocks;
    p.take = take;
    p.run = run < batch->max_q ? run : batch->max_q;
    p.runs = (int)runs;
    return status(attn::launch_cache_fwd_blocks(p, pl, cache->d, cache->page, q->type == ATTN_TYPE_E4M3, static_cast<hipStream_t>(stream)));
}

int attn_fp8_cache_shared_workspace_bytes(const attn_fp8_cache* cache, const attn_fp8_batch* batch, int shared, int Hq,
                                          int max_len, size_t* bytes)
{
    if (!bytes)
        return ATTN_ERR_INVALID_ARG;
    *bytes = 0;
    int st = check_attention(cache, batch, Hq, 1, 1.f, 1.f, max_len);
    attn::SharedPlan pl{};
    if (st == ATTN_OK)
        st = plan_shared(cache, batch, shared, Hq, max_len, pl);
    if (st == ATTN_OK)
        *bytes = pl.pre.bytes + pl.own.bytes;
    return st;
}

int attn_fp8_cache_fwd_shared(const attn_fp8_cache* cache, const attn_fp8_batch* batch, int shared, const attn_fp8_heads* q, int Hq,
                              void* out, int out_type, float* lse, int causal, float sm_scale, float q_descale, int max_len,
                              void* workspace, size_t workspace_bytes, void* stream)
{
    int st = check_attention(cache, batch, Hq, causal, sm_scale, q_descale, max_len);
    if (st != ATTN_OK)
        return st;
    if (!q || (out_type != ATTN_TYPE_BF16 && out_type != ATTN_TYPE_F32) || shared < 0 || shared > batch->W)
        return ATTN_ERR_INVALID_ARG;
    if (batch->B == 0 || batch->T == 0)
        return ATTN_OK;
    if ((st = check_fwd(cache, batch, q, out, lse, workspace)) != ATTN_OK)
        return st;
    attn::SharedPlan pl;
    if ((st = plan_shared(cache, batch, shared, Hq, max_len, pl)) != ATTN_OK)
        return st;
    if (!workspace || workspace_bytes < pl.pre.bytes + pl.own.bytes)
        return ATTN_ERR_INVALID_ARG;
    attn::SharedParams p{};
    fill_fwd(p, cache, batch, q, Hq, out, out_type, lse, causal, sm_scale, q_descale, max_len, workspace);
    p.shared = shared;
    return status(attn::launch_cache_fwd_shared(p, pl, cache->d, cache->page, q->type == ATTN_TYPE_E4M3, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
