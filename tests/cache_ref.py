"""The KV cache's operators on the CPU, in 64 bits, one (sequence, KV head) at a time, from
their definitions; with the bounds that the GPU results are held to.

Nothing here uses the library.  Codes are E4M3 bytes, scales E8M0 bytes."""
from __future__ import annotations

import math

import numpy as np
import torch

import oracle

LOG2E = 1.4426950408889634


def decode(codes):
    """E4M3 bytes -> float64 (0x7F and 0xFF are NaN)."""
    return oracle.e4m3_decode(np.asarray(codes, dtype=np.uint8)).astype(np.float64)


def encode(x):
    """float64, |x| <= 448 or NaN -> E4M3 bytes: nearest, ties to even; by search in the table."""
    table = decode(np.arange(127, dtype=np.uint8))
    a = np.abs(x)
    i = np.clip(np.searchsorted(table, np.where(np.isnan(a), 0, a)), 1, 126)
    lo, hi = table[i - 1], table[i]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 0))
    code = np.where(up, i, i - 1).astype(np.uint8)
    code = np.where(np.isnan(a), 127, code).astype(np.uint8)
    return code | np.where(np.signbit(x) & ~np.isnan(a), 128, 0).astype(np.uint8)


def block_exponent(values):
    """Least e >= -127 with every finite |value| <= 448 2^e."""
    a = np.abs(values[np.isfinite(values)])
    top = float(a.max()) if a.size else 0.0
    e = -127
    while e < 127 and top > 448.0 * 2.0 ** e:
        e += 1
    return e


def rotate(x, table, pos, layout):
    """x [T, H, d] float64, table [n_pos, rot / 2, 2], pos [T]: float64."""
    n_pos, h, _ = table.shape
    y = x.copy()
    for t, p in enumerate(pos):
        cs = table[p].astype(np.float64) if 0 <= p < n_pos else np.full((h, 2), np.nan)
        c, s = cs[:, 0], cs[:, 1]
        ia = np.arange(h) if layout == "half" else 2 * np.arange(h)
        ib = ia + h if layout == "half" else ia + 1
        a, b = x[t][:, ia], x[t][:, ib]
        y[t][:, ia], y[t][:, ib] = a * c - b * s, b * c + a * s
    return y


def tokens(lens, cu, T, b, W, page, max_q):
    """(keys there are, first packed token, new tokens, position of the first)."""
    whole = max(int(lens[b]), 0)
    n = min(whole, W * page)
    if cu is None:
        q = T // len(lens)
        first = b * q
    else:
        first, q = int(cu[b]), int(cu[b + 1]) - int(cu[b])
    return n, first, min(q, max_q), whole - q


class Pages:
    """A cache and its batch as numpy arrays."""

    def __init__(self, k, v, ks, vs, pages, lens):
        self.k, self.v, self.ks, self.vs = (np.array(x) for x in (k, v, ks, vs))
        self.pages, self.lens = np.array(pages), np.array(lens)
        self.n_pages, self.Hkv, self.page, self.d = self.k.shape

    def copy(self):
        return Pages(self.k, self.v, self.ks, self.vs, self.pages, self.lens)

    def page_id(self, b, block):
        p = int(self.pages[b, block]) if block < self.pages.shape[1] else -1
        return p if 0 <= p < self.n_pages else -1

    def keys(self, b, h, which):
        """(codes' values [n, d], exponents [n], there [n]) of a sequence's tokens."""
        n = min(max(int(self.lens[b]), 0), self.pages.shape[1] * self.page)
        c, s = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        x, e, there = np.zeros((n, self.d)), np.zeros(n, dtype=int), np.zeros(n, dtype=bool)
        for j in range(0, n, self.page):
            p, m = self.page_id(b, j // self.page), min(self.page, n - j)
            if p >= 0:
                x[j:j + m], e[j:j + m], there[j:j + m] = decode(c[p, h, :m]), int(s[p, h]) - 127, True
        return x, e, there

    def append(self, k, v, cu=None, max_q=1 << 30, table=None, pos=None, layout="half"):
        """k, v [T, Hkv, d] float64 (exact values of the inputs)."""
        T, W = k.shape[0], self.pages.shape[1]
        for b in range(len(self.lens)):
            n, first, q, pos0 = tokens(self.lens, cu, T, b, W, self.page, max_q)
            lo, end = max(pos0, 0), min(pos0 + q, n)
            kr = k
            if table is not None:
                p = np.asarray(pos) if pos is not None else np.zeros(T, dtype=int)
                if pos is None:
                    p[first:first + q] = pos0 + np.arange(q)
                sel = slice(first, first + q)
                kr = k.copy()
                kr[sel] = rotate(k[sel], table, p[sel], layout)
            for block in range(lo // self.page, (end - 1) // self.page + 1 if end > lo else 0):
                pid = self.page_id(b, block)
                if pid < 0:
                    continue
                t0 = block * self.page
                a, z = max(lo - t0, 0), min(end - t0, self.page)
                for h in range(self.Hkv):
                    for x, c, s in ((kr, self.k, self.ks), (v, self.v, self.vs)):
                        new = x[t0 + a - pos0 + first:t0 + z - pos0 + first, h]
                        new = np.where(np.isfinite(new), new, np.nan)
                        e = block_exponent(new)
                        if a > 0:
                            was = int(s[pid, h]) - 127
                            e = max(e, was)
                            if e > was:
                                c[pid, h, :a] = encode(decode(c[pid, h, :a]) * 2.0 ** (was - e))
                        c[pid, h, a:z] = encode(new * 2.0 ** -e)
                        s[pid, h] = e + 127


def scores(cache, b, h, q, c32):
    """x [rows, keys] (32-bit c, exact products), there [keys]."""
    k, e, there = cache.keys(b, h, "k")
    c = np.float32(c32).astype(np.float64) * 2.0 ** e
    return q @ k.T, c, there


def attention(cache, q, G, cu=None, max_q=1 << 30, causal=True, sm_scale=None, q_descale=1.0):
    """q [T, Hq, d] float64.  Returns out, lse, bound_out, bound_lse [T, Hq, ...] (NaN rows:
    not written).  The bounds, each relative to l:
      - a code whose 2^8 P lies within 2^-19 of the middle between two E4M3 values may be either: x - M
        is rounded once (2^-24 of at most 20), exp2 is within 2 ulp, so P is within 2^-20;
      - the FP8 matrix core adds groups of eight products and drops what lies 13 bits below the
        group's largest: 8 2^-13 of it at most;
      - FP32 sums of n terms: n 2^-24 of the sum of magnitudes, and the same for l."""
    T, Hq, d = q.shape
    W = cache.pages.shape[1]
    sm = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    c32 = np.float32(LOG2E * np.float32(sm).astype(np.float64) * np.float32(q_descale).astype(np.float64))
    out, bound = np.full((T, Hq, d), np.nan), np.full((T, Hq, d), np.nan)
    lse, lbound = np.full((T, Hq), np.nan), np.full((T, Hq), np.nan)
    half = decode(np.arange(127, dtype=np.uint8))
    mid = (half[1:] + half[:-1]) / 2
    for b in range(len(cache.lens)):
        n, first, nq, pos0 = tokens(cache.lens, cu, T, b, W, cache.page, max_q)
        for h in range(cache.Hkv):
            hs = slice(h * G, (h + 1) * G)
            if nq == 0:
                continue
            D, c, there = scores(cache, b, h, q[first:first + nq, hs].reshape(-1, d), c32)
            v, ve, _ = cache.keys(b, h, "v")
            v = v * 2.0 ** ve[:, None]
            i = np.repeat(np.arange(nq), G)
            last = pos0 + i if causal else np.full(nq * G, n - 1)
            see = (np.arange(n)[None] <= last[:, None]) & there[None]
            x = np.where(see, D * c, -np.inf)
            # M from the FP32 product of the largest raw score, as the definition has it
            x32 = np.where(see, (D.astype(np.float32) * c.astype(np.float32)).astype(np.float64), -np.inf)
            pad = -n % 32
            x = np.pad(x, ((0, 0), (0, pad)), constant_values=-np.inf).reshape(nq * G, -1, 32)
            x32 = np.pad(x32, ((0, 0), (0, pad)), constant_values=-np.inf).reshape(nq * G, -1, 32)
            vp = np.pad(v, ((0, pad), (0, 0)))
            r = slice(first, first + nq)
            none = ~see.any(1)
            if n == 0:
                out[r, hs], lse[r, hs], bound[r, hs], lbound[r, hs] = 0, -np.inf, 0, 0
                continue
            M = np.ceil(x32.max(2, keepdims=True))
            M = np.where(np.isfinite(M) | np.isnan(M), M, 0.0)
            m = np.where(none, 0.0, x32.max((1, 2)))[:, None, None]
            y = 256.0 * np.exp2(x - M)
            code = decode(encode(np.minimum(y, 448.0)))
            j = np.clip(np.searchsorted(mid, y), 1, len(mid) - 1)
            near = np.minimum(np.abs(y - mid[j]), np.abs(y - mid[j - 1])) <= 2.0 ** -19 * y
            near &= y > 0
            step = np.where(near, np.maximum(y * 2.0 ** -3, 2.0 ** -9), 0.0)
            lift = np.exp2(M - m)
            p, amb = code * lift / 256, step * lift / 256
            l = np.exp2(x - m).sum((1, 2))
            o = p.reshape(nq * G, -1) @ vp
            pv = p.reshape(nq * G, -1)[:, :, None] * np.abs(vp)[None] if (nq * G * vp.size) < 3e7 else None
            mag = p.reshape(nq * G, -1) @ np.abs(vp)
            if pv is not None:
                trunc = pv.reshape(nq * G, -1, 8, d).max(2).sum(1) * 8 * 2.0 ** -13
            else:
                trunc = mag * 2.0 ** -10
            e = amb.reshape(nq * G, -1) @ np.abs(vp) + trunc + mag * (p.shape[1] + 160) * 2.0 ** -24
            with np.errstate(divide="ignore", invalid="ignore"):
                oo = np.where(none[:, None], 0.0, o / l[:, None])
                ee = np.where(none[:, None], 0.0, e / l[:, None] + np.abs(oo) * 2.0 ** -18)
                ll = np.where(none, -np.inf, math.log(2.0) * (m[:, 0, 0] + np.log2(l)))
            out[r, hs], bound[r, hs] = oo.reshape(nq, G, d), ee.reshape(nq, G, d)
            lse[r, hs] = ll.reshape(nq, G)
            # l within 2^-18 (exp2's 2 ulp, x - M's rounding, the sums); the final FP32 roundings
            lbound[r, hs] = np.where(none, 0.0, 2.0 ** -18 + np.abs(np.where(none, 0, ll)) * 2.0 ** -22).reshape(nq, G)
    return out, lse, bound, lbound


def weights(cache, q, lse, G, n_w, cu=None, max_q=1 << 30, causal=True, sm_scale=None, q_descale=1.0):
    """What cache_weights adds [B, Hkv, n_w] (0 beyond a sequence), lse [T, Hq]; its bound is
    2^-17 of it: x - lse is rounded at magnitudes up to 64 (2^-19), exp2, and the FP32 sum."""
    T, Hq, d = q.shape
    W = cache.pages.shape[1]
    sm = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    c32 = np.float32(LOG2E * np.float32(sm).astype(np.float64) * np.float32(q_descale).astype(np.float64))
    w = np.zeros((len(cache.lens), cache.Hkv, n_w))
    for b in range(len(cache.lens)):
        n, first, nq, pos0 = tokens(cache.lens, cu, T, b, W, cache.page, max_q)
        for h in range(cache.Hkv):
            hs = slice(h * G, (h + 1) * G)
            D, c, there = scores(cache, b, h, q[first:first + nq, hs].reshape(-1, d), c32)
            last = np.repeat(pos0 + np.arange(nq), G) if causal else np.full(nq * G, n - 1)
            see = (np.arange(n)[None] <= last[:, None]) & there[None]
            z = lse[first:first + nq, hs].reshape(-1, 1).astype(np.float64)
            see &= np.isfinite(z)
            x = np.where(see, D * c * math.log(2.0) - np.where(np.isfinite(z), z, 0), -np.inf)
            w[b, h, :n] = np.exp(x).sum(0)[:n]
    return w


def evict(cache, w, budget, n_sink, n_recent, to, new_pages):
    """kept, new_lens, new_weights; writes the pages of `to`."""
    B, Hkv, page = len(cache.lens), cache.Hkv, cache.page
    kept = np.full((B, Hkv, budget), -1, dtype=np.int32)
    nw = np.zeros((B, Hkv, budget), dtype=np.float32)
    lens = np.zeros(B, dtype=np.int32)
    for b in range(B):
        n = min(max(int(cache.lens[b]), 0), cache.pages.shape[1] * page)
        m = lens[b] = min(n, budget)
        for h in range(Hkv):
            ids = list(range(n))
            if n > budget:
                s = min(n_sink, budget)
                r = min(n_recent, budget - s)
                rank = [-math.inf if math.isnan(x) else float(x) for x in w[b, h, :n]]
                isnan = [math.isnan(x) for x in w[b, h, :n]]
                mid = sorted(range(s, n - r), key=lambda t: (isnan[t], -rank[t], t))[:budget - s - r]
                ids = list(range(s)) + sorted(mid) + list(range(n - r, n))
            kept[b, h, :m], nw[b, h, :m] = ids, w[b, h, ids]
            for which, c, sc in (("k", to.k, to.ks), ("v", to.v, to.vs)):
                x, e, _ = cache.keys(b, h, which)
                for j in range(0, m, page):
                    p = int(new_pages[b, j // page])
                    if not 0 <= p < to.n_pages:
                        continue
                    t = ids[j:j + page]
                    y = x[t] * 2.0 ** e[t][:, None]
                    ne = block_exponent(y)
                    c[p, h, :len(t)] = encode(y * 2.0 ** -ne)
                    sc[p, h] = ne + 127
    return kept, lens, nw


# ---- inputs ----

def grid_codes(rng, shape):
    """E4M3 codes of multiples of 2^-3 up to 8 in magnitude: their products with a query on a
    2^-3 grid add up exactly in FP32."""
    x = np.clip(np.round(rng.standard_normal(shape) * 2 * 8) / 8, -8, 8)
    x = np.where(np.abs(x) < 2, np.round(x * 8) / 8, np.where(np.abs(x) < 4, np.round(x * 4) / 4, np.round(x * 2) / 2))
    return encode(x)


def make_cache(rng, B, Hkv, page, d, lens, W=None, spread=2, extra=2):
    """A Pages with shuffled page numbers; unused pages and slots hold NaN codes."""
    W = max(1, max(-(-n // page) for n in lens)) if W is None else W
    used = [-(-n // page) for n in lens]
    total = sum(used) + extra
    k, v = grid_codes(rng, (total, Hkv, page, d)), grid_codes(rng, (total, Hkv, page, d))
    ks = (127 - rng.integers(0, spread + 1, (total, Hkv))).astype(np.uint8)
    vs = (127 + rng.integers(-spread, spread + 1, (total, Hkv))).astype(np.uint8)
    perm = rng.permutation(total)
    pages, at = np.full((B, W), -1, dtype=np.int32), 0
    for b in range(B):
        pages[b, :used[b]] = perm[at:at + used[b]]
        if lens[b] % page:
            last = perm[at + used[b] - 1]
            k[last, :, lens[b] % page:] = 0x7F
            v[last, :, lens[b] % page:] = 0xFF
        at += used[b]
    k[perm[at:]], v[perm[at:]] = 0x7F, 0x7F
    return Pages(k, v, ks, vs, pages, np.array(lens, dtype=np.int32))


def make_queries(rng, T, Hq, d):
    """Queries on a 2^-3 grid that E4M3 and bf16 hold exactly, float64."""
    return decode(grid_codes(rng, (T, Hq, d))) / 4


def torch_q(q, kind):
    t = torch.from_numpy(q).to(torch.bfloat16 if kind == "bf16" else torch.float32)
    return t if kind == "bf16" else t.to(torch.float8_e4m3fn)
