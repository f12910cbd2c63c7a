"""Attention over parts of the E4M3 KV cache, at the sizes it is called with.

Operators: ``bounds`` (least and largest key code of each channel of a page), ``select``
(for every run of queries and KV head the pages whose bounds allow the largest scores),
``blocks`` (attention over the pages of such lists) and ``shared`` (attention of a batch
whose sequences begin with the same pages, read once for all of them).

The cache: ``k``, ``v`` E4M3 codes [pages][Hkv][page][d], ``k_scale``, ``v_scale`` bytes
[pages][Hkv]; a code stands for code * 2^(byte - 127).  Sequence b holds ``lens[b]``
tokens, the new ones among them, in the pages ``table[b]``.  Tokens of a call are packed
[T][heads][d], those of sequence b from ``cu[b]`` on.

Fields of a case: op, B sequences, Hq, Hkv heads, n the longest cache, nq the most new
tokens of a sequence, d, page, ragged (lengths and token counts differ), kind (type of
the queries), take (pages of a list), run (queries of a list), shared (pages that all
sequences begin with).
"""
import math

import torch

own = False

LOG2E = 1.4426950408889634
N_FIRST = 1
N_LAST = 2
E4M3 = torch.float8_e4m3fn
KINDS = {"bf16": torch.bfloat16, "e4m3": E4M3}


def _case(name, op, B, Hq, Hkv, n, nq, d, page, *, ragged=False, kind="bf16", take=0, run=1, shared=0):
    c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, n=n, nq=nq, d=d, page=page, ragged=ragged, kind=kind, take=take, run=run,
             shared=shared)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # after the write of a decode step: the page of each of 16 requests' new token
        _case("bounds_decode_b16_h8_n8192_d128", "bounds", 16, 8, 8, 8192, 1, 128, 128, ragged=True),
        # after the prefill of four prompts: all of their pages
        _case("bounds_prompt_b4_h8_n8192_d128", "bounds", 4, 8, 8, 8192, 8192, 128, 128, ragged=True),
        # a few short requests, small heads and pages: what a call costs at the least
        _case("select_decode_b4_h8kv2_n777_d64", "select", 4, 8, 2, 777, 1, 64, 64, ragged=True, take=4),
        # a decode step of a batch of long contexts: an eighth of each cache
        _case("select_decode_b16_h32kv8_n32768_d128", "select", 16, 32, 8, 32768, 1, 128, 128, take=32),
        # one long-context request in small pages, E4M3 queries
        _case("select_decode_b1_h32kv8_n131001_p64_d128", "select", 1, 32, 8, 131001, 1, 128, 64, kind="e4m3", take=128),
        # the last chunk of a long prompt, a list for every 32 queries
        _case("select_chunk_b1_q2048_h32kv8_n16384_d128", "select", 1, 32, 8, 16384, 2048, 128, 128, take=32, run=32),
        # the attention of the same calls
        _case("blocks_decode_b16_h32kv8_n32768_d128", "blocks", 16, 32, 8, 32768, 1, 128, 128, take=32),
        _case("blocks_decode_b1_h32kv8_n131001_p64_d128", "blocks", 1, 32, 8, 131001, 1, 128, 64, kind="e4m3", take=128),
        _case("blocks_chunk_b1_q2048_h32kv8_n16384_d128", "blocks", 1, 32, 8, 16384, 2048, 128, 128, take=32, run=32),
        # a few requests behind a short common instruction
        _case("shared_decode_b4_h8kv2_n777_d64", "shared", 4, 8, 2, 777, 1, 64, 64, ragged=True, shared=8),
        # decode of a batch that asks about one long document
        _case("shared_decode_b32_h32kv8_s16384_d128", "shared", 32, 32, 8, 17408, 1, 128, 128, ragged=True, shared=128),
        # the questions of such a batch, before the first answer's token: the largest call
        _case("shared_chunk_b8_q192_h32kv8_s16384_d128", "shared", 8, 32, 8, 16576, 192, 128, 128, ragged=True, shared=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of the listed kinds."""
    op = rng.choice(["bounds", "select", "select", "blocks", "blocks", "blocks", "shared", "shared", "shared"])
    d, page = rng.choice([64, 128, 128]), rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 4, 8])
    ragged = rng.random() < 0.6
    kind = rng.choice(["bf16", "bf16", "e4m3"])
    if op == "bounds":
        nq = rng.choice([1, 1, 3, _log(rng, 8, 8192)])
        n = nq + _log(rng, 1, 8192)
        B = _log(rng, 1, max(1, min(64, 32768 // nq)))
        return _case(None, op, min(B, max(1, 400000 // n)), hkv, hkv, n, nq, d, page, ragged=ragged)
    if op == "shared":
        nq = rng.choice([1, 1, 1, 2, _log(rng, 3, 192)])
        shared = _log(rng, 1, 32768 // page)
        n = shared * page + nq + _log(rng, 1, 1024)
        n, nq = n - nq, max(1, min(nq, int(3e8 / (hq * n))))
        n += nq
        B = _log(rng, 2, max(2, min(64, int(6e8 / (hq * nq * n)))))
        return _case(None, op, B, hq, hkv, n, nq, d, page, ragged=ragged, kind=kind, shared=shared)
    nq = rng.choice([1, 1, 1, 2, _log(rng, 8, 2048)])
    run = 1 if nq <= 2 else rng.choice([8, 16, 32, 64])
    n = nq + _log(rng, 1, 131072 if nq <= 2 else 16384)
    take = min(_log(rng, 4, 128), max(4, n // page))
    B = max(1, min(_log(rng, 1, 64), int(2e6 / (hkv * n))))
    if op == "blocks":
        # (the lists' keys and their products: no more than those of the largest listed calls)
        lists = hkv * -(-nq // run)
        most = min((5e5 if run == 1 else 2e6) / (lists * page), 2.6e8 / (hq * nq * page))
        take = max(1, min(take, int(most)))
        B = max(1, min(B, int(most / take)))
    return _case(None, op, B, hq, hkv, n, nq, d, page, ragged=ragged, kind=kind, take=take, run=run)


# ---- inputs ----

def _lengths(case):
    """(lens, new tokens) of the sequences: the first is the longest, the others spread below it."""
    B, n, nq, base = case["B"], case["n"], case["nq"], case["shared"] * case["page"]
    if not case["ragged"]:
        return [n] * B, [nq] * B
    m = n - base
    lens = [max(1, m - (m * 7 * i // (8 * B)) - 13 * i % 29) for i in range(B)]
    if nq == n:
        return lens, list(lens)
    new = [max(1, min(lens[i], nq - (nq * i // (2 * B)) - (i % 3 if nq > 8 else 0))) for i in range(B)]
    return [base + x for x in lens], new


def _pow2(e):
    """2^e in 64 bits for whole e (exp2 and log2 may be off by a rounding)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x):
    """[..., page, d] in 32 bits -> E4M3 codes and bytes, one scale per block."""
    f, t = torch.frexp(x.abs().amax((-2, -1)))
    e = (t - 9 + (f > 0.875).int()).clamp_(min=-127)
    return (x * _pow2(-e).float()[..., None, None]).to(E4M3), (e + 127).to(torch.uint8)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    op, B, Hq, Hkv, d, page = (case[x] for x in ("op", "B", "Hq", "Hkv", "d", "page"))
    lens, new = _lengths(case)
    T = sum(new)
    cu = [0]
    for x in new:
        cu.append(cu[-1] + x)
    st = dict(op=op, page=page, max_q=max(new), take=case["take"], run=case["run"], shared=case["shared"],
              lens=torch.tensor(lens, dtype=torch.int32, device=dev),
              cu=torch.tensor(cu, dtype=torch.int32, device=dev) if case["ragged"] else None)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    # the cache: keys and values of a size that differs from page to page, keys around a middle of
    # their page's own (neighbours speak of the same), one sink key lifted by 7 (the last channel
    # of the queries is 1)
    used = [-(-x // page) for x in lens]
    W, common = max(used), case["shared"]
    total = sum(used) - common * (B - 1)
    k = normal(total, Hkv, page, d).add_(normal(total, Hkv, 1, d)).mul_(torch.exp2(normal(total, Hkv, 1, 1) * 0.5))
    k[..., d - 1] = 0.0
    start = torch.tensor([0] if common else [sum(used[:b]) for b in range(B)], device=dev)
    k[start, :, 0, d - 1] = 7.0 * math.sqrt(d)
    spare = 3
    perm = torch.randperm(total + spare, generator=g, device=dev)
    # (the spare pages and the keys behind a sequence's end hold what an earlier one left)
    cache = []
    for x in (k, None):
        if x is None:
            x = normal(total, Hkv, page, d).mul_(torch.exp2(normal(total, Hkv, 1, 1)))
        code, byte = _quantise(x)
        del x
        c = torch.empty((total + spare, Hkv, page, d), dtype=E4M3, device=dev)
        s = torch.empty((total + spare, Hkv), dtype=torch.uint8, device=dev)
        c.view(torch.uint8)[perm[:total]] = code.view(torch.uint8)
        c.view(torch.uint8)[perm[total:]] = 0x35
        s[perm[:total]], s[perm[total:]] = byte, 127
        cache.append((c, s))
    (kc, ks), (vc, vs) = cache
    st["cache"] = (kc, vc, ks, vs)
    ids, at = perm.cpu().int(), common
    table = torch.full((B, W), -1, dtype=torch.int32)
    for b in range(B):
        table[b, :common] = ids[:common]
        table[b, common:used[b]] = ids[at:at + used[b] - common]
        at += used[b] - common
    st["pages"] = table.to(dev)
    q = normal(T, Hq, d)
    q[..., d - 1] = 1.0
    if op != "bounds":
        st["q"] = q.clamp_(-8, 8).to(KINDS[case["kind"]])
    # the bounds: of the tokens before the new ones where the call is to write them, else of all
    bounds = torch.zeros((total + spare, Hkv, 2, d), dtype=E4M3, device=dev)
    if op == "bounds":
        st["bounds"] = bounds
        _plain_bounds(dict(st, lens=st["lens"] - _counts(st)[1].int()), whole=True)
    elif op != "shared":
        st["bounds"] = bounds
        _plain_bounds(st, whole=True)
    if op == "blocks":
        st["blocks"] = _plain_select(st)
        del st["bounds"]
    return st


# ---- the plain forms ----

def _counts(st):
    """(first new token, new tokens) of each sequence, on the GPU."""
    B = st["lens"].numel()
    if st["cu"] is None:
        return torch.arange(B, device=st["lens"].device) * st["max_q"], torch.full_like(st["lens"], st["max_q"]).long()
    return st["cu"][:-1].long(), (st["cu"][1:] - st["cu"][:-1]).long()


def _plain_bounds(st, whole=False):
    """Of the pages that hold new tokens (whole: all): the least and largest code of each channel,
    rounded outwards to halves."""
    kc, bounds = st["cache"][0], st["bounds"]
    page, dev = st["page"], kc.device
    W = st["pages"].shape[1]
    _, new = _counts(st)
    lens = st["lens"].long()
    old = torch.zeros_like(lens) if whole else lens - new
    blk = torch.arange(W, device=dev)
    touched = (blk * page < lens[:, None]) & ((blk + 1) * page > old[:, None])
    pid = st["pages"].long()[touched]
    there = (lens[:, None] - blk * page)[touched].clamp(max=page)                       # tokens of each page
    for a in range(0, pid.numel(), 2048):
        x = kc[pid[a:a + 2048]].float()                                                 # [pages][Hkv][page][d]
        x = torch.where(torch.isnan(x), 0.0, x)
        has = (torch.arange(page, device=dev) < there[a:a + 2048, None])[:, None, :, None]
        lo = torch.floor(2 * torch.where(has, x, math.inf).amin(2)) / 2
        hi = torch.ceil(2 * torch.where(has, x, -math.inf).amax(2)) / 2
        bounds.view(torch.uint8)[pid[a:a + 2048]] = torch.stack((lo, hi), 2).to(E4M3).view(torch.uint8)
    return bounds


def _runs(st, x, fill):
    """Packed rows [T][...] -> [B][lists][run][...] and the last visible key of each token (-1: none)."""
    first, new = _counts(st)
    n = -(-st["max_q"] // st["run"]) * st["run"]
    i = torch.arange(n, device=x.device)
    valid = i < new[:, None]
    row = (first[:, None] + i).clamp(max=x.shape[0] - 1)
    last = torch.where(valid, (st["lens"].long() - new)[:, None] + i, -1)
    B = last.shape[0]
    y = torch.where(valid.view(B, n, *[1] * (x.dim() - 1)), x[row], fill)
    return y.view(B, -1, st["run"], *x.shape[1:]), last.view(B, -1, st["run"]), valid


def _plain_select(st):
    page, take, bounds, ks = st["page"], st["take"], st["bounds"], st["cache"][2]
    B, W = st["pages"].shape
    Hkv, d, dev = bounds.shape[1], bounds.shape[3], bounds.device
    q, last, _ = _runs(st, st["q"].float(), 0.0)
    _, L, run, Hq, _ = q.shape
    G = Hq // Hkv
    q = q.view(B, L, run, Hkv, G, d).permute(0, 3, 1, 2, 4, 5).reshape(B, Hkv, L * run * G, d)
    # eight bits of each row: whole numbers up to 127 on the row's power of two
    good = torch.isfinite(q).all(-1)
    f, t = torch.frexp(torch.where(good[..., None], q, 0.0).abs().amax(-1))
    e = t - 7 + (f > 0.9921875).int()
    q = torch.round(torch.where(good[..., None], q, 0.0) * _pow2(-e)[..., None].float())
    pid = st["pages"].long()
    x = bounds[pid.clamp(min=0)].float().permute(0, 2, 3, 4, 1)                          # [B][Hkv][2][d][W]
    u = torch.matmul(q.clamp(min=0), x[:, :, 1].contiguous()) + torch.matmul(q.clamp(max=0), x[:, :, 0].contiguous())
    up = e[..., None] + (ks[pid.clamp(min=0)].int() - 127).transpose(1, 2)[:, :, None]
    u = u * _pow2(up.clamp_(-96, 96)).float()
    blk = torch.arange(W, device=dev)
    row_last = last.view(B, 1, L * run, 1).expand(B, Hkv, L * run, G).reshape(B, Hkv, -1, 1)
    u = torch.where(good[..., None] & (blk * page <= row_last), u, -math.inf)
    u = u.view(B, Hkv, L, run * G, W).amax(3).transpose(1, 2)                            # [B][L][Hkv][W]
    seen = last.amax(-1) + 1
    count = ((seen + page - 1) // page)[..., None, None]
    exists = ((blk < count) & (pid >= 0)[:, None, None]).expand(B, L, Hkv, W)
    always = (blk < N_FIRST) | (blk >= count - N_LAST)
    rank = torch.where(always, math.inf, u.clamp(min=-3e38))
    rank = torch.where(exists, rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True)
    best = torch.where(order.values > -math.inf, order.indices, W)[..., :take]
    best = torch.sort(best, dim=-1).values
    best = torch.where(best < W, best, -1).int()
    return torch.nn.functional.pad(best, (0, max(0, take - W)), value=-1).contiguous()


def _partial(x, v):
    """Of scores x [..., rows, keys] in units of log2 (their memory is used) and values [..., keys, d]: the
    row's power of two m, the sum of 2^(x - m), and the sum of the rounded weights times v."""
    top = x.amax(-1, keepdim=True)
    m = torch.ceil(torch.where(top == -math.inf, 0.0, top))
    x = x.view(*x.shape[:-1], -1, 32)
    mg = torch.ceil(x.amax(-1, keepdim=True))
    mg = torch.where(mg == -math.inf, m[..., None], mg)
    p = torch.exp2(x.sub_(mg))
    lift = _pow2((mg - m[..., None]).clamp(min=-900)).float()
    ell = (p.sum(-1, keepdim=True) * lift).sum((-2, -1))
    p = p.mul_(256.0).to(E4M3).float().mul_(lift)
    o = torch.matmul(p.flatten(-2), v) / 256.0
    return torch.where(top == -math.inf, -math.inf, m)[..., 0], ell, o


def _finish(m, ell, o):
    some = ell > 0
    out = torch.where(some[..., None], o / torch.where(some, ell, 1.0)[..., None], 0.0)
    lse = torch.where(some, (m + torch.log2(torch.where(some, ell, 1.0))) * math.log(2.0), -math.inf)
    return out.to(torch.bfloat16), lse


def _values(code, byte, pid, h=None):
    """Pages pid [...] (of head h [...]) in 32 bits."""
    if h is None:
        return code[pid].float() * _pow2(byte[pid].int() - 127).float()[..., None, None]
    return code[pid, h].float() * _pow2(byte[pid, h].int() - 127).float()[..., None, None]


def _plain_blocks(st):
    kc, vc, ks, vs = st["cache"]
    page, blocks = st["page"], st["blocks"].long()
    B, L, Hkv, take = blocks.shape
    T, Hq, d = st["q"].shape
    G, dev = Hq // Hkv, kc.device
    q, last, valid = _runs(st, st["q"].float(), 0.0)
    run = st["run"]
    q = q.view(B, L, run, Hkv, G, d).transpose(2, 3).reshape(B, L, Hkv, run * G, d)
    pid = st["pages"].long()[torch.arange(B, device=dev)[:, None, None, None], blocks.clamp(min=0)]
    listed_ = (blocks >= 0) & (pid >= 0)
    pid, h = pid.clamp(min=0), torch.arange(Hkv, device=dev)[:, None].expand(Hkv, take)
    t = blocks[..., None] * page + torch.arange(page, device=dev)                        # [B][L][Hkv][take][page]
    t = torch.where(listed_[..., None], t, 1 << 40).flatten(-2)
    row_last = last.view(B, L, 1, run, 1).expand(B, L, 1, run, G).reshape(B, L, 1, run * G, 1)
    x = torch.matmul(q, _values(kc, ks, pid, h).flatten(-3, -2).transpose(-2, -1)).mul_(LOG2E / math.sqrt(d))
    x.masked_fill_(t[..., None, :] > row_last, -math.inf)
    out, lse = _finish(*_partial(x, _values(vc, vs, pid, h).flatten(-3, -2)))
    out = out.view(B, L, Hkv, run, G, d).permute(0, 1, 3, 2, 4, 5).reshape(B, L * run, Hq, d)
    lse = lse.view(B, L, Hkv, run, G).permute(0, 1, 3, 2, 4).reshape(B, L * run, Hq)
    return out[valid], lse[valid]


def _plain_shared(st):
    kc, vc, ks, vs = st["cache"]
    page, common = st["page"], st["shared"]
    T, Hq, d = st["q"].shape
    Hkv, dev = kc.shape[1], kc.device
    G, base, scale = Hq // Hkv, common * page, LOG2E / math.sqrt(d)
    # the common pages, all queries at once
    pid = st["pages"][0, :common].long()
    k, v = (_values(c, s, pid).transpose(0, 1).reshape(Hkv, base, d) for c, s in ((kc, ks), (vc, vs)))
    q = st["q"].float().view(T, Hkv, G, d).transpose(0, 1).reshape(Hkv, T * G, d)
    x = torch.matmul(q, k.transpose(-2, -1)).mul_(scale)
    q, last, valid = _runs(st, st["q"].float(), 0.0)
    last = last.flatten(1)
    x.masked_fill_(torch.arange(base, device=dev) > last[valid].repeat_interleave(G)[:, None], -math.inf)
    m1, l1, o1 = (y.view(Hkv, T, G, *y.shape[2:]).transpose(0, 1).flatten(1, 2) for y in _partial(x, v))
    # each sequence's own
    B, W = st["pages"].shape
    pid = st["pages"][:, common:].clamp(min=0).long()
    k, v = (_values(c, s, pid).transpose(1, 2).reshape(B, Hkv, -1, d) for c, s in ((kc, ks), (vc, vs)))
    nq = last.shape[1]
    q = q.reshape(B, nq, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, nq * G, d)
    x = torch.matmul(q, k.transpose(-2, -1)).mul_(scale)
    t = base + torch.arange(k.shape[2], device=dev)
    x.masked_fill_(t > last.repeat_interleave(G, 1)[:, None, :, None], -math.inf)
    m2, l2, o2 = (y.view(B, Hkv, nq, G, *y.shape[3:]).transpose(1, 2).flatten(2, 3)[valid] for y in _partial(x, v))
    m = torch.maximum(m1, m2)
    a, b = (torch.where(y == -math.inf, 0.0, _pow2((y - m).nan_to_num(0.0).clamp(min=-900)).float()) for y in (m1, m2))
    return _finish(m, l1 * a + l2 * b, o1 * a[..., None] + o2 * b[..., None])


def run(state):
    st = state
    op = st["op"]
    if own:
        from paper_2606_06521_amd import attn_fp8 as A
        cache = A.KVCache(*st["cache"])
        if op == "bounds":
            return A.cache_bounds(cache, st["pages"], st["lens"], st["bounds"], cu=st["cu"], max_q=st["max_q"])
        if op == "select":
            return A.cache_select(st["q"], cache, st["pages"], st["lens"], st["bounds"], st["take"], cu=st["cu"],
                                  max_q=st["max_q"], run=st["run"], n_first=N_FIRST, n_last=N_LAST)
        if op == "blocks":
            return A.cache_fwd_blocks(st["q"], cache, st["pages"], st["lens"], st["blocks"], cu=st["cu"],
                                      max_q=st["max_q"], run=st["run"])
        return A.cache_fwd_shared(st["q"], cache, st["pages"], st["lens"], st["shared"], cu=st["cu"], max_q=st["max_q"])
    if op == "bounds":
        return _plain_bounds(st)
    if op == "select":
        return _plain_select(st)
    return _plain_blocks(st) if op == "blocks" else _plain_shared(st)


# ---- what a pass cannot do without ----

def _seen(case):
    """Of each list of a KV head: (tokens of the run, keys that its last one sees)."""
    lens, new = _lengths(case)
    run = case["run"]
    return [(min(run, n - i), m - n + min(i + run, n)) for m, n in zip(lens, new) for i in range(0, n, run)]


def work(case):
    op, Hq, Hkv, d, page, take = (case[x] for x in ("op", "Hq", "Hkv", "d", "page", "take"))
    lens, new = _lengths(case)
    T = sum(new)
    e = KINDS[case["kind"]].itemsize
    pages = sum(-(-x // page) for x in lens)
    if op == "bounds":
        spans = [(x, (x - y) // page * page) for x, y in zip(lens, new)]                # from the first touched page on
        touched = sum(-(-(x - a) // page) for x, a in spans)
        codes = sum(x - a for x, a in spans) * Hkv * d
        return {"bytes": codes + touched * (2 * Hkv * d + 4), "flops": 2.0 * codes}
    if op == "select":
        pairs = sum(n * -(-m // page) for n, m in _seen(case))
        lists = len(_seen(case)) * Hkv
        return {"bytes": pages * (Hkv * (2 * d + 1) + 4) + T * Hq * d * e + 4 * lists * take, "flops": 4.0 * d * Hq * pairs}
    io = T * Hq * (d * (e + 2) + 4)
    if op == "blocks":
        seen = [(n, min(m, take * page)) for n, m in _seen(case)]
        # (what the lists name, or all keys where they name more than there are)
        keys = min(sum(m for _, m in seen), sum(lens))
        return {"bytes": keys * Hkv * 2 * d + 4 * len(seen) * Hkv * take + io, "flops": 4.0 * d * Hq * sum(n * m for n, m in seen)}
    base = case["shared"] * page
    keys = base + sum(x - base for x in lens)
    pairs = sum(n * (m - n) + n * (n + 1) // 2 for m, n in zip(lens, new))
    return {"bytes": keys * Hkv * 2 * d + io, "flops": 4.0 * d * Hq * pairs}


# ---- the same in 64 bits ----

def _exact_bounds(st, new):
    out, page = st["bounds"].clone(), st["page"]
    for b, n in enumerate(st["lens"].tolist()):
        for j in range((n - new[b]) // page, (n - 1) // page + 1):
            p = int(st["pages"][b, j])
            x = st["cache"][0][p, :, :min(page, n - j * page)].double()
            lo, hi = x.min(1).values, x.max(1).values
            lo, hi = -torch.ceil(lo * -2) / 2, -torch.floor(hi * -2) / 2
            out[p, :, 0], out[p, :, 1] = lo.float().to(E4M3), hi.float().to(E4M3)
    return out


def _each_list(st, new):
    """(b, list, first packed token, tokens, position of the first) of every list."""
    at = 0
    for b, n in enumerate(st["lens"].tolist()):
        for i in range(0, new[b], st["run"]):
            yield b, i // st["run"], at + i, min(st["run"], new[b] - i), n - new[b] + i
        at += new[b]


def _exact_select(st, new):
    page, take = st["page"], st["take"]
    B, W = st["pages"].shape
    Hkv, d = st["bounds"].shape[1], st["bounds"].shape[3]
    G = st["q"].shape[1] // Hkv
    out = torch.full((B, -(-st["max_q"] // st["run"]), Hkv, take), -1, dtype=torch.int32)
    for b, i, at, n, pos in _each_list(st, new):
        nb = (pos + n - 1) // page + 1
        p = st["pages"][b, :nb].long()
        start = torch.arange(nb, device=p.device) * page
        last = torch.arange(pos, pos + n, device=p.device).repeat_interleave(G)
        for h in range(Hkv):
            q = st["q"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, d)
            top = q.abs().amax(1)
            e = torch.ceil(torch.log2(top / 127.0).clamp(min=-300))
            e = torch.where(top > 127.0 * _pow2(e), e + 1, torch.where(top <= 127.0 * _pow2(e - 1), e - 1, e))
            q = torch.round(q / _pow2(e)[:, None])
            lo, hi = (st["bounds"][p, h, w].double() for w in (0, 1))
            up = (e[:, None] + st["cache"][2][p, h].double() - 127).clamp(-96, 96)
            s = torch.empty((n * G, nb), dtype=torch.float64, device=p.device)
            step = max(1, (1 << 25) // (nb * d))
            for r in range(0, n * G, step):
                s[r:r + step] = torch.maximum(q[r:r + step, None] * lo, q[r:r + step, None] * hi).sum(2)
            s = (s * _pow2(up)).masked_fill(start > last[:, None], -math.inf).amax(0).tolist()
            must = set(range(min(N_FIRST, nb))) | set(range(max(0, nb - N_LAST), nb))
            ids = sorted(range(nb), key=lambda j: (j not in must, -s[j], j))[:take]
            out[b, i, h, :len(ids)] = torch.tensor(sorted(ids), dtype=torch.int32)
    return out


def _weighted(z, v):
    """Rows of scores z in natural units (-inf: not seen), values v: out and lse, weights rounded in groups of 32."""
    s = torch.logsumexp(z, 1)
    x = torch.nn.functional.pad(z * math.log2(math.e), (0, -z.shape[1] % 32), value=-math.inf).view(z.shape[0], -1, 32)
    top = torch.ceil(x.amax(2, keepdim=True)).clamp(min=-1e300)
    y = 256 * torch.exp2(x - top)
    quantum = _pow2((torch.frexp(y).exponent - 1).clamp(min=-6) - 3)
    y = torch.round(y / quantum) * quantum / 256 * torch.exp2(top - (s * math.log2(math.e))[:, None, None])
    return y.flatten(1)[:, :z.shape[1]] @ v, s


def _exact_rows(st, new, lists):
    """Attention by sequence, KV head and list (or run of 512 queries over all keys)."""
    T, Hq, d = st["q"].shape
    Hkv, page, dev = st["cache"][0].shape[1], st["page"], st["q"].device
    G = Hq // Hkv
    out = torch.zeros((T, Hq, d), dtype=torch.float64, device=dev)
    lse = torch.zeros((T, Hq), dtype=torch.float64, device=dev)
    blocks = st["blocks"].tolist() if lists else None
    for b, i, at, n, pos in _each_list(st if lists else dict(st, run=512), new):
        for h in range(Hkv):
            ids = [j for j in blocks[b][i][h] if j >= 0] if lists else range((pos + n - 1) // page + 1)
            ids = torch.tensor(list(ids), device=dev)
            p = st["pages"][b].long()[ids]
            t = (ids[:, None] * page + torch.arange(page, device=dev)).flatten()
            k, v = ((c[p, h].double() * _pow2(s[p, h].int() - 127)[:, None, None]).flatten(0, 1)
                    for c, s in ((st["cache"][0], st["cache"][2]), (st["cache"][1], st["cache"][3])))
            q = st["q"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, d)
            z = q @ k.T.contiguous() / math.sqrt(d)
            z = z.masked_fill(t > torch.arange(pos, pos + n, device=dev).repeat_interleave(G)[:, None], -math.inf)
            o, s = _weighted(z, v)
            out[at:at + n, h * G:(h + 1) * G], lse[at:at + n, h * G:(h + 1) * G] = o.view(n, G, d), s.view(n, G)
    return out, lse


def exact(case, seed):
    if case["op"] == "select" and case["B"] * case["Hkv"] * -(-case["nq"] // case["run"]) > 4096:
        return None
    st = prepare(case, seed)
    _, new = _lengths(case)
    if case["op"] == "bounds":
        return _exact_bounds(st, new)
    if case["op"] == "select":
        return _exact_select(st, new)
    return _exact_rows(st, new, case["op"] == "blocks")
