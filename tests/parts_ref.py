"""Attention over parts of the KV cache on the CPU, in 64 bits, from the definitions; with the bounds
that the GPU results are held to.  Caches and batches are those of cache_ref.  Nothing here uses the
library but for its plans (host code), so that a test can say which kernel it runs."""
from __future__ import annotations

import ctypes
import math

import numpy as np

from tests import cache_ref as R
from tests.cache_plan import Plan


# ---- plans ----

class SharedPlan(ctypes.Structure):
    """attn::SharedPlan"""
    _fields_ = [("pre", Plan), ("own", Plan)]


def _lib():
    from paper_2606_06521_amd import attn_fp8
    return ctypes.CDLL(attn_fp8.LIB_PATH)


def blocks_plan(lists, G, run, take, page, d, n_cu=256):
    f = _lib()["_ZN4attn11blocks_planEliiiiii"]
    f.argtypes, f.restype = [ctypes.c_int64] + [ctypes.c_int] * 6, Plan
    return f(lists, G, run, take, page, d, n_cu)


def shared_plan(B, Hkv, G, T, max_q, shared, max_len, page, d, n_cu=256):
    f = _lib()["_ZN4attn11shared_planEiiiiiiiiii"]
    f.argtypes, f.restype = [ctypes.c_int] * 10, SharedPlan
    return f(B, Hkv, G, T, max_q, shared, max_len, page, d, n_cu)


# ---- bounds ----

def bounds(cache, given, cu=None, max_q=1 << 30):
    """given float64 [n_pages, Hkv, 2, d]: the same with the touched pages' bounds."""
    out, W, page = given.copy(), cache.pages.shape[1], cache.page
    T = 0 if cu is not None else len(cache.lens) * max_q
    for b in range(len(cache.lens)):
        n, _, q, pos0 = R.tokens(cache.lens, cu, T, b, W, page, max_q)
        lo, end = max(pos0, 0), min(pos0 + q, n)
        for block in range(lo // page, (end - 1) // page + 1 if end > lo else 0):
            p = cache.page_id(b, block)
            if p < 0:
                continue
            x = R.decode(cache.k[p, :, :min(end - block * page, page)])
            x = np.where(np.isnan(x), 0.0, x)
            out[p, :, 0], out[p, :, 1] = np.floor(2 * x.min(1)) / 2, np.ceil(2 * x.max(1)) / 2
    return out


# ---- choice ----

def eight_bits(q):
    """Rows q [..., d] as whole numbers and exponents; rows that are not finite as zeros, and which those are."""
    bad = ~np.isfinite(q).all(-1)
    q = np.where(bad[..., None], 0.0, q)
    top = np.abs(q).max(-1)
    f, t = np.frexp(top)
    e = t - 7 + (f > 127 / 128)
    return np.round(q * np.exp2(-e.astype(np.float64))[..., None]), e, bad


def runs_of(cache, b, cu, T, max_q, run):
    """(list, first packed token, tokens, position of the first), keys there are."""
    n, first, q, pos0 = R.tokens(cache.lens, cu, T, b, cache.pages.shape[1], cache.page, max_q)
    return [(i // run, first + i, min(run, q - i), pos0 + i) for i in range(0, q, run)], n


def last_seen(pos, m, G, n, causal):
    """Last visible key of each row of a run."""
    at = pos + np.repeat(np.arange(m), G)
    return np.where(at < 0, -1, np.minimum(at, n - 1) if causal else n - 1)


def select(cache, q, bnds, G, take, run=1, n_first=1, n_last=1, cu=None, max_q=None, causal=True, max_len=0):
    """q [T, Hq, d] float64 (may hold infinities and NaN), bnds [n_pages, Hkv, 2, d]."""
    T, _, d = q.shape
    B, page = len(cache.lens), cache.page
    max_q = T // B if max_q is None else max_q
    out = np.full((B, -(-max_q // run), cache.Hkv, take), -1, dtype=np.int32)
    for b in range(B):
        lists, n = runs_of(cache, b, cu, T, max_q, run)
        n = min(n, max_len) if max_len else n
        for i, at, m, pos in lists:
            last = last_seen(pos, m, G, n, causal)
            nb = last[-1] // page + 1
            for h in range(cache.Hkv):
                rows, e, bad = eight_bits(q[at:at + m, h * G:(h + 1) * G].reshape(m * G, d))
                keys = []
                for j in range(nb):
                    p = cache.page_id(b, j)
                    if p < 0:
                        continue
                    must = j < n_first or j >= nb - n_last
                    use = ~bad & (last >= j * page)
                    s = -math.inf
                    if use.any():
                        u = np.maximum(rows * bnds[p, h, 0], rows * bnds[p, h, 1]).sum(1)
                        s = (u * np.exp2(np.clip(e + int(cache.ks[p, h]) - 127, -96, 96).astype(np.float64)))[use].max()
                    keys.append((not must, -s, j))
                ids = sorted(j for _, _, j in sorted(keys)[:take])
                out[b, i, h, :len(ids)] = ids
    return out


# ---- attention ----

def weighted(q, k, c, see, v):
    """Rows q [rows, d], codes' values k, v [keys, d], score factors c [keys], which are seen: out, lse and their
    bounds (as in cache_ref.attention, where they are derived).  keys is a multiple of 32.  A NaN of a key makes
    NaN of the rows that see it, one of a value of its channel there (bounds 0); others get nothing of it."""
    bad_k = np.isnan(k).any(1)
    poisoned = (see & bad_k).any(1) | np.isnan(q).any(1) & see.any(1)
    hit = (see.astype(np.float64) @ np.isnan(v).astype(np.float64) > 0) | poisoned[:, None]
    k, v = np.where(np.isnan(k), 0.0, k), np.where(np.isnan(v), 0.0, v)
    D = np.where(np.isnan(q), 0.0, q) @ k.T
    half = R.decode(np.arange(127, dtype=np.uint8))
    mid = (half[1:] + half[:-1]) / 2
    rows, n = D.shape
    d = v.shape[1]
    x = np.where(see, D * c, -np.inf).reshape(rows, -1, 32)
    x32 = np.where(see, (D.astype(np.float32) * c.astype(np.float32)).astype(np.float64), -np.inf).reshape(rows, -1, 32)
    none = ~see.any(1)
    M = np.ceil(x32.max(2, keepdims=True))
    M = np.where(np.isfinite(M) | np.isnan(M), M, 0.0)
    m = np.where(none, 0.0, x32.max((1, 2)))[:, None, None]
    y = 256.0 * np.exp2(x - M)
    code = R.decode(R.encode(np.minimum(y, 448.0)))
    j = np.clip(np.searchsorted(mid, y), 1, len(mid) - 1)
    near = (np.minimum(np.abs(y - mid[j]), np.abs(y - mid[j - 1])) <= 2.0 ** -19 * y) & (y > 0)
    step = np.where(near, np.maximum(y * 2.0 ** -3, 2.0 ** -9), 0.0)
    lift = np.exp2(M - m)
    p, amb = (code * lift / 256).reshape(rows, -1), (step * lift / 256).reshape(rows, -1)
    l = np.exp2(x - m).sum((1, 2))
    o, mag = p @ v, p @ np.abs(v)
    if p.size * d < 3e7:
        trunc = (p[:, :, None] * np.abs(v)[None]).reshape(rows, -1, 8, d).max(2).sum(1) * 8 * 2.0 ** -13
    else:
        trunc = mag * 2.0 ** -10
    e = amb @ np.abs(v) + trunc + mag * (n + 160) * 2.0 ** -24
    with np.errstate(divide="ignore", invalid="ignore"):
        out = np.where(none[:, None], 0.0, o / l[:, None])
        bound = np.where(none[:, None], 0.0, e / l[:, None] + np.abs(out) * 2.0 ** -18)
        lse = np.where(none, -np.inf, math.log(2.0) * (m[:, 0, 0] + np.log2(l)))
    lbound = np.where(none, 0.0, 2.0 ** -18 + np.abs(np.where(none, 0, lse)) * 2.0 ** -22)
    return np.where(hit, np.nan, out), np.where(poisoned, np.nan, lse), np.where(hit, 0.0, bound), np.where(poisoned, 0.0, lbound)


def attention(cache, q, blocks, G, run=1, cu=None, max_q=None, causal=True, sm_scale=None, q_descale=1.0):
    """Over the blocks [B, runs, Hkv, take] alone (None: over all there are); results as cache_ref.attention's,
    bounds that are NaN: not written."""
    T, Hq, d = q.shape
    B, page = len(cache.lens), cache.page
    max_q = T // B if max_q is None else max_q
    if blocks is None:
        W = cache.pages.shape[1]
        blocks = np.broadcast_to(np.arange(W), (B, -(-max_q // run), cache.Hkv, W))
    sm = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    c32 = np.float32(R.LOG2E * np.float32(sm).astype(np.float64) * np.float32(q_descale).astype(np.float64))
    out, bound = np.full((T, Hq, d), np.nan), np.full((T, Hq, d), np.nan)
    lse, lbound = np.full((T, Hq), np.nan), np.full((T, Hq), np.nan)
    for b in range(B):
        lists, n = runs_of(cache, b, cu, T, max_q, run)
        for i, at, m, pos in lists:
            last = last_seen(pos, m, G, n, causal)
            for h in range(cache.Hkv):
                ids = [(int(j), cache.page_id(b, int(j))) for j in blocks[b, i, h] if 0 <= j]
                ids = [(j, p) for j, p in ids if p >= 0 and j * page < n]
                r, hs = slice(at, at + m), slice(h * G, (h + 1) * G)
                if not ids:
                    out[r, hs], lse[r, hs], bound[r, hs], lbound[r, hs] = 0, -np.inf, 0, 0
                    continue
                t = np.concatenate([j * page + np.arange(page) for j, _ in ids])
                k = np.concatenate([R.decode(cache.k[p, h]) for _, p in ids])
                v = np.concatenate([R.decode(cache.v[p, h]) * 2.0 ** (int(cache.vs[p, h]) - 127) for _, p in ids])
                c = np.repeat([c32.astype(np.float64) * 2.0 ** (int(cache.ks[p, h]) - 127) for _, p in ids], page)
                k, v = np.where((t < n)[:, None], k, 0.0), np.where((t < n)[:, None], v, 0.0)
                o, s, e, f = weighted(q[r, hs].reshape(m * G, d), k, c, t[None] <= last[:, None], v)
                out[r, hs], bound[r, hs] = o.reshape(m, G, d), e.reshape(m, G, d)
                lse[r, hs], lbound[r, hs] = s.reshape(m, G), f.reshape(m, G)
    return out, lse, bound, lbound


def share(cache, n_shared):
    """All sequences begin with sequence 0's first pages (which are full in all that are long enough)."""
    cache.pages[1:, :n_shared] = cache.pages[0, :n_shared]
    return cache
