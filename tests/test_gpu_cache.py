"""The KV cache's operators on the GPU against 64-bit results (tests/cache_ref.py): rotary
positions, append, attention, weights, eviction, and a run of them together."""
import math

import numpy as np
import pytest
import torch

from tests import cache_ref as R
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# half a unit in the last place, relative
HALF = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}


@pytest.fixture(scope="module")
def A():
    from paper_2606_06521_amd import attn_fp8
    return attn_fp8


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def dev_cache(A, c):
    return A.KVCache(dev(c.k).view(torch.float8_e4m3fn), dev(c.v).view(torch.float8_e4m3fn), dev(c.ks), dev(c.vs))


def same_cache(got, want):
    for name, g, w in zip("k v k_scale v_scale".split(), got, (want.k, want.v, want.ks, want.vs)):
        g = g.view(torch.uint8).cpu().numpy()
        # (a NaN is a NaN, and 0 has two codes)
        if name in "kv":
            g, w = np.where(g & 127 == 127, 127, g), np.where(w & 127 == 127, 127, w)
            g, w = np.where(g == 128, 0, g), np.where(w == 128, 0, w)
        bad = np.argwhere(g != w)
        assert bad.size == 0, (name, len(bad), bad[:4].tolist(), [(int(g[tuple(i)]), int(w[tuple(i)])) for i in bad[:4]])


def within(got, want, tol):
    """|got - want| <= tol everywhere."""
    over = np.abs(got - want) - tol
    i = np.unravel_index(np.argmax(np.where(np.isnan(over), np.inf, over)), over.shape)
    assert over[i] <= 0, (i, float(got[i]), float(want[i]), float(over[i]))


def cu_of(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


# ---- rope ----

@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,H,d,rot", [(1, 1, 16, 16), (3, 5, 64, 32), (130, 3, 128, 128), (7, 2, 80, 48)])
def test_rope(A, T, H, d, rot, kind, layout):
    log(f"rope T={T} H={H} d={d} rot={rot} {kind} {layout}")
    g = torch.Generator().manual_seed(T + d)
    x = torch.randn((T, H + 2, d), generator=g).to(TYPES[kind])
    table = A.rope_table(977, rot, device="cpu")
    pos = torch.randint(0, 977, (T,), generator=g, dtype=torch.int32)
    view = x.cuda()[:, 1:H + 1]                      # heads in the middle of wider rows
    out = A.rope(view, table.cuda(), pos.cuda(), layout=layout)
    xs = x[:, 1:H + 1].double().numpy()
    want = R.rotate(xs, table.numpy(), pos.numpy(), layout)
    # a c - b s in FP32: each product and the sum round once, 2^-24 of |a c| + |b s| each
    # (with all signs made positive one of the two channels is the sum of magnitudes, with sin's negative the other)
    mag = np.abs(R.rotate(np.abs(xs), np.abs(table.numpy()) * [1, -1], pos.numpy(), layout)) + \
        np.abs(R.rotate(np.abs(xs), np.abs(table.numpy()), pos.numpy(), layout))
    tol = HALF[kind] * np.abs(want) + 3 * 2.0 ** -24 * mag + 2.0 ** -25 * (kind == "fp16")
    within(out.cpu().double().numpy(), want, tol)
    # in place, and the neighbours stay
    y = x.cuda()
    A.rope(y[:, 1:H + 1], table.cuda(), pos.cuda(), layout=layout, out=y[:, 1:H + 1])
    assert torch.equal(y[:, 1:H + 1], out) and torch.equal(y[:, 0].cpu(), x[:, 0]) and torch.equal(y[:, -1].cpu(), x[:, -1])


def test_rope_positions_outside_the_table_are_nan(A):
    x = torch.randn((4, 2, 64)).cuda()
    pos = torch.tensor([-1, 0, 9, 10], dtype=torch.int32).cuda()
    out = A.rope(x, A.rope_table(10, 32), pos)
    assert torch.isnan(out[[0, 3], :, :32]).all() and torch.equal(out[..., 32:], x[..., 32:])
    assert torch.isfinite(out[1:3]).all()


# ---- append ----

CASES_APPEND = [
    # lens after the call, new tokens
    ([1], [1]), ([64], [1]), ([65, 1, 128], [1, 1, 1]), ([200, 129, 64], [3, 129, 64]), ([300, 257], [300, 2]),
    ([7, 0, 130], [7, 0, 1]),
]


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("case", range(len(CASES_APPEND)))
def test_append(A, case, d, page, kind):
    lens, new = CASES_APPEND[case]
    Hkv, Hq, rot = 2, 4, d // 2 if case % 2 else d
    layout = "interleaved" if case % 3 == 1 else "half"
    log(f"append {lens} {new} d={d} page={page} {kind}")
    rng = np.random.default_rng(case * 7 + d)
    c = R.make_cache(rng, len(lens), Hkv, page, d, lens)
    T, cu = sum(new), cu_of(new)
    t = torch.from_numpy(rng.standard_normal((T + 3, Hq + 2 * Hkv, d)) * np.exp2(rng.integers(-6, 7, (T + 3, 1, 1)))).to(TYPES[kind])
    table = A.rope_table(max(max(lens), 1), rot, device="cpu")
    gc = dev_cache(A, c)
    x = t.cuda()
    q_out = torch.full((T + 3, Hq, d), 5.0, dtype=TYPES[kind], device="cuda")
    # (three tokens behind the last sequence: read by nobody, their rows of q_out stay)
    A.cache_append(gc, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], dev(c.pages), dev(c.lens), cu=dev(cu), max_q=max(new),
                   table=table.cuda(), layout=layout, q=x[:, :Hq], q_out=q_out)
    full = t.double().numpy()
    c.append(full[:, Hq:Hq + Hkv], full[:, Hq + Hkv:], cu=cu, table=table.numpy(), layout=layout)
    same_cache(gc, c)
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, new)]).astype(int)
    want = R.rotate(full[:T, :Hq], table.numpy(), pos, layout)
    got = q_out.cpu().double().numpy()
    # (FP32 as in test_rope; subnormal fp16 values are 2^-24 apart)
    within(got[:T], want, HALF[kind] * np.abs(want) + 2.0 ** -22 * np.abs(full[:T, :Hq]).max(-1, keepdims=True) + 2.0 ** -25 * (kind == "fp16"))
    assert np.all(got[T:] == 5.0)


def test_append_token_by_token_without_rotation(A):
    """The scale of a block grows with its tokens; older codes follow it."""
    rng = np.random.default_rng(11)
    lens = np.array([0, 61], dtype=np.int32)
    c = R.make_cache(rng, 2, 2, 64, 64, [140, 200])
    c.lens = lens
    gc = dev_cache(A, c)
    for step in range(70):
        log(f"append step {step}")
        c.lens = c.lens + 1
        t = torch.from_numpy(rng.standard_normal((2, 2, 2, 64)) * 2.0 ** (step % 9 - 4)).bfloat16()
        A.cache_append(gc, t[0].cuda(), t[1].cuda(), dev(c.pages), dev(c.lens))
        c.append(t[0].double().numpy(), t[1].double().numpy())
    same_cache(gc, c)


def test_append_values_that_are_not_finite_and_zero_blocks(A):
    rng = np.random.default_rng(3)
    c = R.make_cache(rng, 2, 1, 64, 64, [3, 2])
    t = torch.from_numpy(rng.standard_normal((2, 5, 1, 64))).float()
    t[0, 1, 0, 5], t[0, 2, 0, 6], t[1, 0, 0, 7] = float("inf"), float("nan"), float("-inf")
    t[0, 3:] = 0.0
    t[1, 3:] = 1e-42
    gc = dev_cache(A, c)
    A.cache_append(gc, t[0].cuda(), t[1].cuda(), dev(c.pages), dev(c.lens), cu=dev(cu_of([3, 2])), max_q=3)
    c.append(t[0].double().numpy(), t[1].double().numpy(), cu=cu_of([3, 2]))
    same_cache(gc, c)
    assert int(gc.k_scale[int(c.pages[1, 0]), 0]) == 0


def test_append_leaves_out_what_has_no_place(A):
    """No page, tokens before position 0, more tokens than max_q, cu entries past T."""
    rng = np.random.default_rng(4)
    lens, new = [130, 5, 70], [130, 9, 70]
    c = R.make_cache(rng, 3, 2, 64, 64, lens)
    c.pages[0, 1] = c.n_pages          # out of range
    c.pages[2, 0] = -7
    T = sum(new)
    t = torch.from_numpy(rng.standard_normal((2, T, 2, 64))).bfloat16()
    gc = dev_cache(A, c)
    cu = cu_of(new)
    A.cache_append(gc, t[0].cuda(), t[1].cuda(), dev(c.pages), dev(c.lens), cu=dev(cu), max_q=129)
    c.append(t[0].double().numpy(), t[1].double().numpy(), cu=cu, max_q=129)
    same_cache(gc, c)


# ---- attention ----

def run_fwd(A, c, q, G, kind, new=None, causal=True, check=True, max_len=0, out_dtype=torch.float32, **kw):
    T, Hq, d = q.shape
    cu = None if new is None else cu_of(new)
    max_q = T // len(c.lens) if new is None else max(max(new), 1)
    gq = R.torch_q(q, kind).cuda()
    out = torch.full((T, Hq, d), 7.0, dtype=out_dtype, device="cuda")
    lse = torch.full((T, Hq), 7.0, device="cuda")
    gc = dev_cache(A, c)
    A.cache_fwd(gq, gc, dev(c.pages), dev(c.lens), cu=None if cu is None else dev(cu), max_q=max_q, causal=causal,
                max_len=max_len, out=out, lse=lse, **kw)
    if not check:
        return out, lse, None
    want, wl, bound, lb = R.attention(c, q, G, cu=cu, max_q=max_q, causal=causal, **kw)
    o, l = out.cpu().double().numpy(), lse.cpu().double().numpy()
    left = np.isnan(bound)
    assert np.all(o[left] == 7.0) and np.all(l[np.isnan(lb)] == 7.0)
    o, w, b = o[~left], want[~left], bound[~left]
    if out_dtype == torch.bfloat16:
        b = b + np.abs(w) * 2.0 ** -8
    within(o, w, b)
    l, w, b = l[~np.isnan(lb)], wl[~np.isnan(lb)], lb[~np.isnan(lb)]
    assert np.array_equal(np.isinf(l), np.isinf(w))
    if np.isfinite(w).any():
        within(l[np.isfinite(w)], w[np.isfinite(w)], b[np.isfinite(w)])
    return out, lse, want


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("lens", [[1], [127, 128, 129, 0], [2000, 31, 700], [65, 64, 63, 33, 32]])
def test_fwd_decode(A, lens, d, page, kind):
    G, Hkv = 4, 2
    log(f"fwd decode {lens} d={d} page={page} {kind}")
    rng = np.random.default_rng(len(lens) + d)
    c = R.make_cache(rng, len(lens), Hkv, page, d, lens)
    q = R.make_queries(rng, len(lens), G * Hkv, d)
    run_fwd(A, c, q, G, kind)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,page,G", [(64, 128, 1), (64, 64, 3), (128, 64, 8), (128, 128, 4)])
@pytest.mark.parametrize("lens,new", [([40], [40]), ([300, 129, 5], [17, 129, 5]), ([500, 0, 260, 128], [1, 0, 33, 100]),
                                      ([1000, 90], [200, 3])])
def test_fwd_chunk(A, lens, new, d, page, G, causal):
    Hkv = 2
    log(f"fwd chunk {lens} {new} d={d} page={page} G={G} causal={causal}")
    rng = np.random.default_rng(sum(lens) + d + G)
    c = R.make_cache(rng, len(lens), Hkv, page, d, lens)
    q = R.make_queries(rng, sum(new) + 2, G * Hkv, d)     # two rows behind the last sequence
    run_fwd(A, c, q, G, "bf16" if G != 3 else "e4m3", new=new, causal=causal)


@pytest.mark.parametrize("n", [3000, 16500])
def test_fwd_split_over_keys(A, n):
    """Few rows and many keys: ranges, and their merge; a short and an empty sequence beside them."""
    rng = np.random.default_rng(n)
    lens = [n, 140, 0, 1]
    c = R.make_cache(rng, 4, 1, 128, 128, lens)
    q = R.make_queries(rng, 4, 5, 128)
    log(f"fwd split n={n}")
    st, nbytes = A.attn_fp8_cache_workspace_bytes(A.attn_fp8_cache(None, None, None, None, c.n_pages, 1, 128, 128),
                                                  A.attn_fp8_batch(None, None, None, 4, c.pages.shape[1], 4, 1), 5, 0)
    assert st == 0 and nbytes > 0
    run_fwd(A, c, q, 5, "bf16")
    run_fwd(A, c, q, 5, "e4m3", out_dtype=torch.bfloat16)


def test_fwd_scales_descales_and_a_far_maximum(A):
    """Block scales over their range, a q descale, scores whose maximum comes late and far above."""
    rng = np.random.default_rng(8)
    c = R.make_cache(rng, 2, 2, 64, 64, [700, 450])
    c.ks[:] = rng.integers(118, 133, c.ks.shape)
    c.vs[:] = rng.choice([60, 100, 127, 180], c.vs.shape)
    q = R.make_queries(rng, 2, 4, 64)
    run_fwd(A, c, q, 2, "e4m3", q_descale=0.75, sm_scale=0.25)


def test_fwd_pages_that_are_none_are_not_seen(A):
    rng = np.random.default_rng(9)
    c = R.make_cache(rng, 3, 2, 64, 128, [400, 129, 64])
    c.pages[0, 2], c.pages[1, 2], c.pages[2, 0] = -1, 1 << 30, c.n_pages
    q = R.make_queries(rng, 6, 4, 128)
    log("fwd bad pages")
    _, lse, _ = run_fwd(A, c, q, 2, "bf16", new=[3, 2, 1])
    assert torch.isinf(lse[5]).all()                     # its only page is none


def test_fwd_lengths_outside_the_table(A):
    rng = np.random.default_rng(10)
    c = R.make_cache(rng, 3, 1, 64, 64, [128, 128, 100])
    c.lens = np.array([1000, -5, 100], dtype=np.int32)
    run_fwd(A, c, R.make_queries(rng, 3, 2, 64), 2, "bf16")
    # max_len cuts too
    c.lens = np.array([90, 64, 30], dtype=np.int32)
    q = R.make_queries(rng, 3, 2, 64)
    _, _, want = run_fwd(A, c, q, 2, "bf16", max_len=90)
    c.lens = np.array([100, 64, 30], dtype=np.int32)
    out, _, _ = run_fwd(A, c, q, 2, "bf16", max_len=90, check=False)
    assert np.allclose(out.cpu().numpy(), want, atol=2e-2)


def test_fwd_queries_with_strides(A):
    rng = np.random.default_rng(12)
    c = R.make_cache(rng, 2, 2, 128, 128, [300, 77])
    q = R.make_queries(rng, 2, 8, 128)
    wide = torch.zeros((2, 16, 128), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:11] = R.torch_q(q, "bf16").cuda()
    gc = dev_cache(A, c)
    o1, l1 = A.cache_fwd(wide[:, 3:11], gc, dev(c.pages), dev(c.lens))
    o2, l2 = A.cache_fwd(R.torch_q(q, "bf16").cuda(), gc, dev(c.pages), dev(c.lens))
    assert torch.equal(o1, o2) and torch.equal(l1, l2)
    turned = R.torch_q(q, "bf16").cuda().transpose(0, 1).contiguous().transpose(0, 1)   # heads outermost
    o3, l3 = A.cache_fwd(turned, gc, dev(c.pages), dev(c.lens))
    assert torch.equal(o3, o2) and torch.equal(l3, l2)


# ---- weights ----

@pytest.mark.parametrize("d,page,G,kind", [(64, 64, 2, "e4m3"), (64, 128, 1, "bf16"), (128, 64, 4, "bf16"), (128, 128, 8, "e4m3")])
@pytest.mark.parametrize("lens,new,causal", [([1], [1], True), ([300, 0, 129], [1, 0, 1], True), ([500, 90, 64], [37, 90, 64], True),
                                             ([260, 33], [20, 3], False), ([18000, 300], [70, 90], True)])
def test_weights(A, lens, new, causal, d, page, G, kind):
    Hkv = 2
    log(f"weights {lens} {new} d={d} page={page} G={G} {kind}")
    rng = np.random.default_rng(sum(lens) + d)
    c = R.make_cache(rng, len(lens), Hkv, page, d, lens)
    cu, T = cu_of(new), sum(new)
    q = R.make_queries(rng, T, G * Hkv, d)
    lse = R.attention(c, q, G, cu=cu, causal=causal)[1].astype(np.float32)
    n_w = c.pages.shape[1] * page + 5
    start = rng.random((len(lens), Hkv, n_w)).astype(np.float32)
    w = dev(start)
    A.cache_weights(R.torch_q(q, kind).cuda(), dev(lse), dev_cache(A, c), dev(c.pages), dev(c.lens), w, cu=dev(cu),
                    max_q=max(new), causal=causal)
    want = R.weights(c, q, lse, G, n_w, cu=cu, causal=causal)
    got = w.cpu().double().numpy()
    # the sum's own rounding (2^-24 of the result), and 2^-17 of what is added (cache_ref)
    within(got, start + want, 2.0 ** -17 * want + 2.0 ** -24 * (start + want))
    assert np.array_equal(got[want == 0], start[want == 0].astype(np.float64))


# ---- eviction ----

@pytest.mark.parametrize("d,page", [(64, 64), (128, 128), (128, 64), (64, 128)])
@pytest.mark.parametrize("lens,budget,n_sink,n_recent", [([1], 1, 0, 0), ([300, 129, 0, 64], 100, 4, 32), ([1500, 900], 200, 4, 0),
                                                         ([300], 10, 20, 5), ([300], 10, 4, 30), ([200, 40], 130, 0, 130), ([2500], 2499, 4, 16)])
def test_evict(A, lens, budget, n_sink, n_recent, d, page):
    Hkv, B = 2, len(lens)
    log(f"evict {lens} budget={budget} sink={n_sink} recent={n_recent} d={d} page={page}")
    rng = np.random.default_rng(sum(lens) + budget)
    c = R.make_cache(rng, B, Hkv, page, d, lens, spread=12)
    n_w = c.pages.shape[1] * page
    # few distinct values (ties), zeros of both signs, negative ones, NaN, infinities
    w = np.round(rng.standard_normal((B, Hkv, n_w)) * 4).astype(np.float32)
    flat = w.reshape(-1)
    flat[rng.integers(0, flat.size, 9)] = np.nan
    flat[rng.integers(0, flat.size, 3)] = np.inf
    flat[rng.integers(0, flat.size, 3)] = -np.inf
    flat[rng.integers(0, flat.size, 9)] = -0.0
    nb = -(-budget // page)
    to = R.make_cache(rng, B, Hkv, page, d, [nb * page] * B)
    new_pages = to.pages.copy()
    gt = dev_cache(A, to)
    kept, new_lens, nw = A.cache_evict(dev_cache(A, c), dev(c.pages), dev(c.lens), dev(w), gt, dev(new_pages), budget,
                                       n_sink=n_sink, n_recent=n_recent)
    wk, wl, ww = R.evict(c, w, budget, n_sink, n_recent, to, new_pages)
    assert np.array_equal(kept.cpu().numpy(), wk)
    assert np.array_equal(new_lens.cpu().numpy(), wl)
    assert np.array_equal(nw.cpu().numpy(), ww, equal_nan=True)
    same_cache(gt, to)


def test_evict_within_one_cache_and_bad_pages(A):
    rng = np.random.default_rng(21)
    c = R.make_cache(rng, 2, 1, 64, 64, [200, 150], extra=5)
    spare = [p for p in range(c.n_pages) if p not in c.pages]
    new_pages = np.array([[spare[0], spare[1]], [c.n_pages + 3, spare[2]]], dtype=np.int32)
    w = rng.random((2, 1, c.pages.shape[1] * 64)).astype(np.float32)
    gc = dev_cache(A, c)
    kept, lens, _ = A.cache_evict(gc, dev(c.pages), dev(c.lens), dev(w), gc, dev(new_pages), 100, n_sink=2, n_recent=8)
    to = c.copy()
    wk, wl, _ = R.evict(c, w, 100, 2, 8, to, new_pages)
    assert np.array_equal(kept.cpu().numpy(), wk) and np.array_equal(lens.cpu().numpy(), wl)
    same_cache(gc, to)


# ---- together ----

def serve(A, table, cache, pages, lens, qkv, Hq, Hkv, w, cu, max_q):
    """One step as a server makes it: append, attend, weigh."""
    q = A.cache_append(cache, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], pages, lens, cu=cu, max_q=max_q, table=table, q=qkv[:, :Hq])
    out, lse = A.cache_fwd(q, cache, pages, lens, cu=cu, max_q=max_q)
    A.cache_weights(q, lse, cache, pages, lens, w, cu=cu, max_q=max_q)
    return q, out, lse


def test_prompt_decode_evict_decode(A):
    """A ragged prompt, decode steps, an eviction to new pages, and more decode steps: the cache's
    bytes, the kept tokens and every output against the 64-bit run on the same q."""
    B, Hq, Hkv, d, page, budget = 2, 4, 2, 64, 64, 96
    rng = np.random.default_rng(31)
    c = R.make_cache(rng, B, Hkv, page, d, [5 * page] * B, extra=8)
    c.lens = np.array([150, 70], dtype=np.int32)
    spare = [p for p in range(c.n_pages) if p not in c.pages]
    gc = dev_cache(A, c)
    table = A.rope_table(1024, d)
    tab = table.cpu().numpy()
    w = torch.zeros((B, Hkv, 5 * page), device="cuda")
    wr = np.zeros((B, Hkv, 5 * page))

    def step(new, pos):
        T, cu = sum(new), cu_of(new)
        x = torch.from_numpy(rng.standard_normal((T, Hq + 2 * Hkv, d))).bfloat16()
        q, out, lse = serve(A, table, gc, dev(c.pages), dev(c.lens), x.cuda(), Hq, Hkv, w, dev(cu), max(new))
        f = x.double().numpy()
        c.append(f[:, Hq:Hq + Hkv], f[:, Hq + Hkv:], cu=cu, table=tab)
        qr = q.cpu().double().numpy()
        want, wl, bound, lb = R.attention(c, qr, Hq // Hkv, cu=cu)
        # (scores of values off the grid: FP32 sums of 128 products of at most 64, 2^-13 in a score of either sign)
        within(out.cpu().double().numpy(), want, bound + np.abs(want) * 2.0 ** -8 + 2e-2)
        within(lse.cpu().double().numpy(), wl, lb + 2.0 ** -13)
        got = R.weights(c, qr, lse.cpu().numpy(), Hq // Hkv, wr.shape[2], cu=cu)
        wr.__iadd__(got)
        within(w.cpu().double().numpy(), wr, 2e-3 * wr + 1e-6)

    log("prompt")
    step([150, 70], None)
    for i in range(3):
        log(f"decode {i}")
        c.lens = c.lens + 1
        step([1, 1], None)
    same_cache(gc, c)
    log("evict")
    new_pages = np.array(spare[:4], dtype=np.int32).reshape(2, 2)
    before = w.cpu().numpy()
    kept, lens, nw = A.cache_evict(gc, dev(c.pages), dev(c.lens), w, gc, dev(new_pages), budget, n_recent=16)
    to = c.copy()
    wk, wl, ww = R.evict(c, before, budget, 4, 16, to, new_pages)
    assert np.array_equal(kept.cpu().numpy(), wk) and np.array_equal(lens.cpu().numpy(), wl)
    c = to
    c.lens = wl
    c.pages = np.concatenate([new_pages, np.array(spare[4:6], dtype=np.int32).reshape(2, 1)], 1)
    same_cache(gc, c)
    w = torch.zeros((B, Hkv, 3 * page), device="cuda")
    w[:, :, :budget] = nw
    wr = w.cpu().double().numpy()
    for i in range(2):
        log(f"decode after {i}")
        c.lens = c.lens + 1
        step([1, 1], None)
    same_cache(gc, c)


def test_captured_step_follows_the_lengths(A):
    """A decode step captured once and replayed while lens grows, beside eager work, equals eager steps."""
    B, Hq, Hkv, d, page = 3, 4, 2, 128, 128
    rng = np.random.default_rng(41)
    c = R.make_cache(rng, B, Hkv, page, d, [20 * page] * B)
    start = np.array([1500, 127, 3], dtype=np.int32)
    table = A.rope_table(20 * page, d)
    pages = dev(c.pages)
    xs = [torch.randn((B, Hq + 2 * Hkv, d), device="cuda").bfloat16() for _ in range(4)]
    eager, lens = [], dev(start)
    ge = dev_cache(A, c)
    we = torch.zeros((B, Hkv, 20 * page), device="cuda")
    for x in xs:
        lens = lens + 1
        _, out, lse = serve(A, table, ge, pages, lens, x, Hq, Hkv, we, None, 1)
        eager.append((out.clone(), lse.clone()))
    gg = dev_cache(A, c)
    wg = torch.zeros_like(we)
    lens, x = dev(start + 1), xs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve(A, table, gg, pages, lens, x, Hq, Hkv, torch.zeros_like(wg), None, 1)     # warm
    torch.cuda.current_stream().wait_stream(side)
    gg = dev_cache(A, c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, out, lse = serve(A, table, gg, pages, lens, x, Hq, Hkv, wg, None, 1)
    for i, xi in enumerate(xs):
        log(f"replay {i}")
        x.copy_(xi)
        lens.copy_(dev(start + 1 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i][0]) and torch.equal(lse, eager[i][1])
        serve(A, table, ge, pages, lens, x, Hq, Hkv, torch.zeros_like(we), None, 1)      # eager work between
    assert torch.equal(wg, we)


def test_calls_on_another_stream(A):
    rng = np.random.default_rng(51)
    c = R.make_cache(rng, 2, 2, 128, 128, [5000, 700])
    q = R.torch_q(R.make_queries(rng, 2, 8, 128), "bf16").cuda()
    gc, pages, lens = dev_cache(A, c), dev(c.pages), dev(c.lens)
    want, wl = A.cache_fwd(q, gc, pages, lens)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out, lse = A.cache_fwd(q, gc, pages, lens, stream=s)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl)


# ---- values that are not finite ----

@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 20), (128, 64, 1, 130), (64, 128, 8, 40)])
def test_fwd_nan_values_reach_the_rows_that_see_them(A, d, page, G, new):
    """NaN codes of K and V in a chunk: rows before them are as without, rows from them on are NaN (V: in
    the NaN's channel alone)."""
    rng = np.random.default_rng(d + new)
    n = 150 + new
    c = R.make_cache(rng, 1, 1, page, d, [n])
    q = R.make_queries(rng, new, G, d)
    want, wl, bound, lb = R.attention(c, q, G)
    t = n - new // 2                                   # a key that the first half of the rows does not see
    pid, slot = int(c.pages[0, t // page]), t % page
    log(f"nan d={d} page={page} G={G} new={new}")
    first = t - (n - new)                              # the first row that sees it
    c.v[pid, 0, slot, 5] = 0x7F
    c.v[pid, 0, slot, d - 1] = 0xFF
    out, lse, _ = run_fwd(A, c, q, G, "bf16", check=False)
    o, l = out.cpu().double().numpy(), lse.cpu().double().numpy()
    hit = np.zeros(o.shape, dtype=bool)
    hit[first:, :, [5, d - 1]] = True
    assert np.array_equal(np.isnan(o), hit)
    within(np.where(hit, 0, o), np.where(hit, 0, want), bound)
    within(l, wl, lb)
    # a NaN in K: the rows that see it have a NaN score
    c.k[pid, 0, slot, 3] = 0x7F
    out, lse, _ = run_fwd(A, c, q, G, "bf16", check=False)
    o, l = out.cpu().double().numpy(), lse.cpu().double().numpy()
    assert np.isnan(o[first:]).all() and np.isnan(l[first:]).all()
    within(o[:first], want[:first], bound[:first])
    within(l[:first], wl[:first], lb[:first])


def test_fwd_queries_that_are_not_finite_stay_in_their_rows(A):
    rng = np.random.default_rng(77)
    c = R.make_cache(rng, 2, 1, 64, 64, [300, 90])
    q = R.make_queries(rng, 2, 4, 64)
    want, wl, bound, lb = R.attention(c, q, 4)
    t = R.torch_q(q, "bf16")
    t[0, 1, 7], t[0, 2, 3], t[1, 0, 0] = float("nan"), float("inf"), float("-inf")
    out, lse = A.cache_fwd(t.cuda(), dev_cache(A, c), dev(c.pages), dev(c.lens), out_dtype=torch.float32)
    o, l = out.cpu().double().numpy(), lse.cpu().double().numpy()
    bad = np.zeros((2, 4), dtype=bool)
    bad[0, 1] = bad[0, 2] = bad[1, 0] = True
    assert np.isnan(o[bad]).all() and np.isnan(l[bad]).all()
    within(o[~bad], want[~bad], bound[~bad])
    within(l[~bad], wl[~bad], lb[~bad])


@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 1), (128, 64, 4, 130), (64, 128, 8, 40)])
def test_factors_below_fp32_leave_masked_keys_out(A, d, page, G, new):
    """Blocks of zeros (scale 2^-127) and a small descale: the factor of their scores lies below FP32's
    least value, the scores are 0, and keys that a row does not see get nothing."""
    rng = np.random.default_rng(d + G)
    n = 200 + new
    c = R.make_cache(rng, 1, 1, page, d, [n])
    c.k[:], c.ks[:] = 0, 0
    q = R.make_queries(rng, new, G, d)
    log(f"small factor d={d} page={page} G={G} new={new}")
    _, lse, _ = run_fwd(A, c, q, G, "bf16", sm_scale=2.0 ** -10, q_descale=2.0 ** -30)
    w = torch.zeros((1, 1, c.pages.shape[1] * page), device="cuda")
    A.cache_weights(R.torch_q(q, "bf16").cuda(), lse, dev_cache(A, c), dev(c.pages), dev(c.lens), w, sm_scale=2.0 ** -10,
                    q_descale=2.0 ** -30)
    want = R.weights(c, q, lse.cpu().numpy(), G, w.shape[2], sm_scale=2.0 ** -10, q_descale=2.0 ** -30)
    within(w.cpu().double().numpy(), want, 2.0 ** -17 * want)


@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 1), (128, 64, 4, 130), (64, 128, 8, 40)])
def test_fwd_scores_beyond_two_to_the_thirty(A, d, page, G, new):
    """Scores so large that FP32 has no fraction for them: the softmax of their FP32 values, whose
    differences are 0 or far above 30, so a row's result is the mean of the values of its largest keys.
    Its bound: the matrix core's 8 2^-13 of the largest product; lse is M ln 2 in FP32, two roundings
    and log2 of a count."""
    rng = np.random.default_rng(3 * d + G)
    n = 260 + new
    c = R.make_cache(rng, 1, 1, page, d, [n])
    c.ks[:] = rng.choice([163, 167, 171], c.ks.shape)
    q = R.make_queries(rng, new, G, d)
    q[::3] = -np.abs(q[::3])                            # with the keys of some blocks all positive: all scores
    c.k[c.pages[0, 0]] &= 0x7F                          # of a block, or nearly, below 0
    log(f"far scores d={d} page={page} G={G} new={new}")
    out, lse, _ = run_fwd(A, c, q, G, "bf16", check=False)
    c32 = np.float32(R.LOG2E * np.float32(1 / math.sqrt(d)).astype(np.float64))
    D, cf, _ = R.scores(c, 0, 0, q.reshape(-1, d), c32)
    assert np.array_equal(D, D.astype(np.float32))
    x = (D.astype(np.float32) * cf.astype(np.float32)).astype(np.float64)
    see = np.arange(n)[None] <= np.repeat(n - new + np.arange(new), G)[:, None]
    x = np.where(see, x, -np.inf)
    top = x.max(1, keepdims=True)
    others = np.where(x == top, -np.inf, x).max(1)
    assert (np.abs(top) > 2.0 ** 30).all() and (top[:, 0] - others > 64).all()
    v, ve, _ = R.Pages.keys(c, 0, 0, "v")
    v = v * 2.0 ** ve[:, None]
    p = (x == top) / (x == top).sum(1, keepdims=True)
    o, l = out.cpu().double().numpy().reshape(-1, d), lse.cpu().double().numpy().reshape(-1)
    within(o, p @ v, np.broadcast_to(2.0 ** -10 * np.abs(v).max(), o.shape))
    wl = (top[:, 0] + np.log2((x == top).sum(1))) * math.log(2.0)
    within(l, wl, 2.0 ** -22 * np.abs(wl))


# ---- sizes and arguments at the edges ----

def test_cache_beyond_four_gigabytes(A):
    """Pages whose bytes lie past 2^32 of the arrays: append, attention, weights, eviction."""
    rng = np.random.default_rng(91)
    Hkv, page, d, n_pages = 8, 128, 128, 40000
    c = R.make_cache(rng, 2, Hkv, page, d, [300, 140], extra=4)
    # the small cache's pages at the end of a large one
    big = [torch.empty((n_pages, Hkv, page, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((n_pages, Hkv), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    at = n_pages - c.n_pages
    log(f"cache of {big[0].numel() / 2 ** 30:.1f} GiB")
    assert at * Hkv * page * d > 1 << 32
    for x, y in zip(big + scales, (c.k, c.v, c.ks, c.vs)):
        x[at:] = dev(y)
    gc = A.KVCache(*big, *scales)
    pages = dev(np.where(c.pages >= 0, c.pages + at, -1).astype(np.int32))

    def same():
        same_cache([x[at:] for x in gc], c)

    t = torch.from_numpy(rng.standard_normal((2, 2, Hkv, d))).bfloat16()
    c.lens = c.lens + 1
    A.cache_append(gc, t[0].cuda(), t[1].cuda(), pages, dev(c.lens))
    c.append(t[0].double().numpy(), t[1].double().numpy())
    same()
    q = R.make_queries(rng, 2, Hkv, d)
    out, lse = A.cache_fwd(R.torch_q(q, "bf16").cuda(), gc, pages, dev(c.lens), out_dtype=torch.float32)
    want, wl, bound, lb = R.attention(c, q, 1)
    # (the appended tokens are off the grid: their scores round to FP32)
    within(out.cpu().double().numpy(), want, bound + 2e-4)
    within(lse.cpu().double().numpy(), wl, lb + 1e-5)
    w = torch.zeros((2, Hkv, pages.shape[1] * page), device="cuda")
    A.cache_weights(R.torch_q(q, "bf16").cuda(), lse, gc, pages, dev(c.lens), w)
    ww = R.weights(c, q, lse.cpu().numpy(), 1, w.shape[2])
    within(w.cpu().double().numpy(), ww, 2.0 ** -16 * ww + 1e-12)
    spare = np.array([p for p in range(c.n_pages) if p not in c.pages][:2], dtype=np.int32).reshape(2, 1)
    kept, _, _ = A.cache_evict(gc, pages, dev(c.lens), w, gc, dev(spare + at), 100)
    wk, _, _ = R.evict(c, w.cpu().numpy(), 100, 4, 0, c, spare)
    assert np.array_equal(kept.cpu().numpy(), wk)
    same()


def test_token_offsets_outside_the_call(A):
    """cu entries past T or in disorder: what lies inside is done, nothing outside is touched."""
    rng = np.random.default_rng(92)
    c = R.make_cache(rng, 3, 2, 64, 64, [70, 40, 9])
    q = R.make_queries(rng, 5, 4, 64)
    inside = np.array([0, 3, 5, 5], dtype=np.int32)
    for cu in ([0, 3, 99, 1 << 30], [-4, 3, 5, 2]):
        cu = np.array(cu, dtype=np.int32)
        log(f"cu {cu.tolist()}")
        out = torch.full((5, 4, 64), 7.0, device="cuda")
        lse = torch.full((5, 4), 7.0, device="cuda")
        A.cache_fwd(R.torch_q(q, "bf16").cuda(), dev_cache(A, c), dev(c.pages), dev(c.lens), cu=dev(cu), max_q=5, out=out, lse=lse)
        want, wl, bound, lb = R.attention(c, q, 2, cu=inside)
        within(out.cpu().double().numpy(), want, bound)
        within(lse.cpu().double().numpy(), wl, lb)


def test_strides_of_single_tokens_and_heads_are_not_looked_at(A):
    rng = np.random.default_rng(93)
    c = R.make_cache(rng, 1, 1, 64, 64, [50])
    q = R.torch_q(R.make_queries(rng, 1, 1, 64), "bf16").cuda()
    odd = torch.as_strided(q, (1, 1, 64), (3, 5, 1))
    args = dev_cache(A, c), dev(c.pages), dev(c.lens)
    assert torch.equal(A.cache_fwd(odd, *args)[0], A.cache_fwd(q, *args)[0])
    t, pos = A.rope_table(8, 64), torch.tensor([3], dtype=torch.int32, device="cuda")
    assert torch.equal(A.rope(odd, t, pos), A.rope(q, t, pos))


def test_binding_refuses_what_does_not_fit(A):
    """Checked before the library is called; nothing is launched."""
    rng = np.random.default_rng(94)
    c = R.make_cache(rng, 2, 2, 64, 64, [70, 40])
    gc, pages, lens = dev_cache(A, c), dev(c.pages), dev(c.lens)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((2, 2, 128), device="cuda")
    lse = torch.zeros((2, 4), device="cuda")
    table, pos = A.rope_table(128, 64), torch.zeros(2, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    bad = [
        lambda: A.cache_fwd(q.float(), gc, pages, lens), lambda: A.cache_fwd(q[:, :3], gc, pages, lens),
        lambda: A.cache_fwd(q[..., :32], gc, pages, lens), lambda: A.cache_fwd(q, gc, pages.long(), lens),
        lambda: A.cache_fwd(q, gc, pages, lens[:1]), lambda: A.cache_fwd(q, gc, pages, lens, cu=cu),
        lambda: A.cache_fwd(q, gc, pages, lens, cu=cu[:2], max_q=1), lambda: A.cache_fwd(q, gc, pages, lens, max_q=0),
        lambda: A.cache_fwd(q, gc, pages, lens, out=torch.empty((2, 4, 32), device="cuda")),
        lambda: A.cache_fwd(q, gc, pages, lens, lse=lse.double()), lambda: A.cache_fwd(q, gc._replace(v=gc.k[:1]), pages, lens),
        lambda: A.cache_fwd(q, gc._replace(k_scale=gc.k_scale[:, :1]), pages, lens),
        lambda: A.cache_fwd(q.cpu(), gc, pages, lens), lambda: A.cache_fwd(q, gc._replace(k=gc.k.cpu()), pages, lens),
        lambda: A.cache_fwd(q.repeat(2, 1, 1)[:3], gc, pages, lens),
        lambda: A.cache_append(gc, k, k[:, :1], pages, lens), lambda: A.cache_append(gc, k, k.half(), pages, lens),
        lambda: A.cache_append(gc, k, k, pages, lens, q=q), lambda: A.cache_append(gc, k, k, pages, lens, table=table, q=q[:1]),
        lambda: A.cache_append(gc, k, k, pages, lens, table=table.double()),
        lambda: A.cache_append(gc, k, k, pages, lens, table=table, positions=pos.long()),
        lambda: A.cache_weights(q, lse, gc, pages, lens, w[:, :, :100]), lambda: A.cache_weights(q, lse[:1], gc, pages, lens, w),
        lambda: A.cache_weights(q, lse, gc, pages, lens, w.double()),
        lambda: A.cache_weights(q, lse, gc, pages, lens, w[:1].expand(2, 2, 128)),
        lambda: A.cache_evict(gc, pages, lens, w, gc, pages, 64), lambda: A.cache_evict(gc, pages, lens, w, gc, pages[:, :1], 0),
        lambda: A.cache_evict(gc, pages, lens, w, A.kv_cache(4, 2, 64, page=128), pages[:, :1].contiguous(), 64),
        lambda: A.rope(q, table, pos.long()), lambda: A.rope(q, table[..., 0], pos), lambda: A.rope(q[0], table, pos),
        lambda: A.rope(q, table, pos, out=q[:1]), lambda: A.rope(q.double(), table, pos),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
    for call in (lambda: A.cache_fwd(q, gc, pages, lens, sm_scale=0.0), lambda: A.cache_fwd(q, gc, pages, lens, max_len=-1),
                 lambda: A.rope(q, A.rope_table(8, 8), pos), lambda: A.cache_append(gc, k, k, pages, lens, table=A.rope_table(8, 24))):
        with pytest.raises(A.AttnError):
            call()
    with pytest.raises(KeyError):
        A.rope(q, table, pos, layout="other")


def test_tokens_past_the_page_table_have_no_place(A):
    """lens past W * page: the tokens that fit are written where they belong, no older one is overwritten;
    queries of the others see every key there is."""
    rng = np.random.default_rng(95)
    c = R.make_cache(rng, 2, 2, 64, 64, [128, 128])
    c.lens = np.array([129, 131], dtype=np.int32)          # 1 past the table; 3 past it, one inside
    new = [1, 4]
    t = torch.from_numpy(rng.standard_normal((2, 5, 2, 64))).bfloat16()
    gc, cu = dev_cache(A, c), cu_of(new)
    A.cache_append(gc, t[0].cuda(), t[1].cuda(), dev(c.pages), dev(c.lens), cu=dev(cu), max_q=4)
    before = c.copy()
    c.append(t[0].double().numpy(), t[1].double().numpy(), cu=cu, max_q=4)
    same_cache(gc, c)
    assert np.array_equal(c.k[c.pages[0]], before.k[before.pages[0]])
    c = before
    q = R.make_queries(rng, 5, 4, 64)
    run_fwd(A, c, q, 2, "bf16", new=new)
    lse = R.attention(c, q, 2, cu=cu)[1].astype(np.float32)
    w = torch.zeros((2, 2, 128), device="cuda")
    A.cache_weights(R.torch_q(q, "bf16").cuda(), dev(lse), dev_cache(A, c), dev(c.pages), dev(c.lens), w, cu=dev(cu), max_q=4)
    want = R.weights(c, q, lse, 2, 128, cu=cu)
    within(w.cpu().double().numpy(), want, 2.0 ** -17 * want)


def test_largest_values_survive_append_and_eviction(A):
    """Values next to FP32's largest: 2^128 after rounding, as codes and scales."""
    c = R.make_cache(np.random.default_rng(96), 1, 1, 64, 64, [3])
    x = torch.full((3, 1, 64), 1.0)
    x[0, 0, 5], x[1, 0, 6], x[2, 0, 7] = 3.4e38, -3.3e38, 1e38
    gc = dev_cache(A, c)
    A.cache_append(gc, x.cuda(), x.cuda(), dev(c.pages), dev(c.lens))
    c.append(x.double().numpy(), x.double().numpy())
    same_cache(gc, c)
    to, new_pages = c.copy(), np.array([[c.n_pages - 1 if c.pages[0, 0] != c.n_pages - 1 else 0]], dtype=np.int32)
    w = torch.tensor([[[1.0, 2.0, 0.0] + [0.0] * 61]]).cuda()
    A.cache_evict(gc, dev(c.pages), dev(c.lens), w, gc, dev(new_pages), 2, n_sink=0)
    R.evict(c, w.cpu().numpy(), 2, 0, 0, to, new_pages)
    same_cache(gc, to)


def test_two_streams_and_two_graphs_at_once(A):
    """Split calls (each with a workspace of its own) side by side on two streams, and two captured ones
    replayed in turn: all equal the calls by themselves."""
    rng = np.random.default_rng(97)
    sets = []
    for n in (9000, 5000):
        c = R.make_cache(rng, 2, 2, 128, 128, [n, 300])
        args = (R.torch_q(R.make_queries(rng, 2, 8, 128), "bf16").cuda(), dev_cache(A, c), dev(c.pages), dev(c.lens))
        st, nbytes = A.attn_fp8_cache_workspace_bytes(A.attn_fp8_cache(None, None, None, None, c.n_pages, 2, 128, 128),
                                                      A.attn_fp8_batch(None, None, None, 2, c.pages.shape[1], 2, 1), 8, 0)
        assert st == 0 and nbytes > 0
        sets.append((args, A.cache_fwd(*args)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[A.cache_fwd(*args, stream=s) for _ in range(8)] for (args, _), s in zip(sets, streams)]
    torch.cuda.synchronize()
    for (_, want), calls in zip(sets, got):
        for o, l in calls:
            assert torch.equal(o, want[0]) and torch.equal(l, want[1])
    graphs = []
    for args, want in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = A.cache_fwd(*args)
        graphs.append((g, r, want))
    for i in range(4):
        log(f"replay {i}")
        for g, r, want in graphs:
            r[0].fill_(3.0)
            g.replay()
        A.cache_fwd(*sets[0][0])
        torch.cuda.synchronize()
        for _, r, want in graphs:
            assert torch.equal(r[0], want[0]) and torch.equal(r[1], want[1])


def test_every_call_on_another_stream(A):
    """The whole step on a stream of its own, behind work that is still running there."""
    rng = np.random.default_rng(98)
    B, Hq, Hkv, d, page = 2, 4, 2, 64, 64
    c = R.make_cache(rng, B, Hkv, page, d, [200, 100], extra=6)
    spare = np.array([p for p in range(c.n_pages) if p not in c.pages][:4], dtype=np.int32).reshape(2, 2)
    x = torch.from_numpy(rng.standard_normal((B, Hq + 2 * Hkv, d))).bfloat16().cuda()
    table, pages, lens, new_pages = A.rope_table(256, d), dev(c.pages), dev(c.lens), dev(spare)

    def step(stream):
        gc = dev_cache(A, c)
        w = torch.zeros((B, Hkv, pages.shape[1] * page), device="cuda")
        late = torch.zeros_like(x)
        torch.cuda.synchronize()
        if stream is None:
            late.copy_(x)
        else:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)       # the inputs arrive late on that stream
                late.copy_(x)
        kw = dict(stream=stream)
        q = A.cache_append(gc, late[:, Hq:Hq + Hkv], late[:, Hq + Hkv:], pages, lens, table=table, q=late[:, :Hq], **kw)
        r = A.rope(late[:, :Hq], table, torch.tensor([199, 99], dtype=torch.int32, device="cuda") if stream is None else pos, **kw)
        out, lse = A.cache_fwd(q, gc, pages, lens, **kw)
        A.cache_weights(q, lse, gc, pages, lens, w, **kw)
        kept, nl, nw = A.cache_evict(gc, pages, lens, w, gc, new_pages, 100, **kw)
        torch.cuda.synchronize()
        return [q, r, out, lse, w, kept, nl, nw, *(t.view(torch.uint8) for t in gc)]

    pos = torch.tensor([199, 99], dtype=torch.int32, device="cuda")
    for a, b in zip(step(None), step(torch.cuda.Stream())):
        assert torch.equal(a, b)
