"""Attention over parts of the KV cache on the GPU against 64-bit results (tests/parts_ref.py): bounds
of pages, choice of pages, attention over lists and behind a shared prefix, and a run of them."""
import math

import numpy as np
import pytest
import torch

from tests import cache_ref as R
from tests import parts_ref as P
from tests.gpu_helpers import log
from tests.test_gpu_cache import cu_of, dev, dev_cache, within

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def A():
    from paper_2606_06521_amd import attn_fp8
    return attn_fp8


def n_cu():
    return torch.cuda.get_device_properties(0).multi_processor_count


def dev_bounds(x):
    """float64 E4M3 values -> codes on the GPU."""
    return dev(R.encode(x)).view(E4M3)


def values(t):
    return R.decode(t.view(torch.uint8).cpu().numpy())


# ---- bounds ----

CASES_BOUNDS = [([1], [1]), ([64, 65, 129, 300], [1, 1, 1, 1]), ([200, 129, 64, 0], [3, 129, 64, 0]), ([700, 257], [700, 130]),
                ([60, 10], [70, 10])]


@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("case", range(len(CASES_BOUNDS)))
def test_bounds(A, case, d, page):
    lens, new = CASES_BOUNDS[case]
    log(f"bounds {lens} {new} d={d} page={page}")
    rng = np.random.default_rng(case * 5 + d + page)
    c = R.make_cache(rng, len(lens), 3, page, d, lens)
    # any codes, NaN and both zeros among them
    c.k = rng.integers(0, 256, c.k.shape, dtype=np.uint8)
    given = R.decode(rng.integers(0, 120, (c.n_pages, 3, 2, d), dtype=np.uint8))
    got = dev_bounds(given)
    r = A.cache_bounds(dev_cache(A, c), dev(c.pages), dev(c.lens), got, cu=dev(cu_of(new)), max_q=max(new))
    assert r is got
    want = P.bounds(c, given, cu=cu_of(new), max_q=max(new))
    assert np.array_equal(values(got), want)
    assert not (got.view(torch.uint8).cpu().numpy() == 0x80).any()


@pytest.mark.parametrize("max_q", [None, 1, 5, 128, 129])
def test_bounds_of_the_last_tokens(A, max_q):
    rng = np.random.default_rng(3)
    lens = [300, 2, 128, 0, 257]
    c = R.make_cache(rng, 5, 2, 64, 128, lens)
    given = np.full((c.n_pages, 2, 2, 128), 1.5)
    got = dev_bounds(given)
    A.cache_bounds(dev_cache(A, c), dev(c.pages), dev(c.lens), got, max_q=max_q)
    # (a sequence shorter than max_q begins before position 0)
    n = c.pages.shape[1] * 64 if max_q is None else max_q
    assert np.array_equal(values(got), P.bounds(c, given, max_q=n))


def test_bounds_of_small_and_large_codes(A):
    """Every code by itself: rounded outwards to halves."""
    c = R.make_cache(np.random.default_rng(4), 1, 2, 64, 128, [64])
    codes = np.array([x for x in range(256) if x & 127 != 127], dtype=np.uint8)
    c.k[c.pages[0, 0]] = codes[:128][None, None]
    c.k[c.pages[0, 0], 1] = codes[126:][None]
    got = A.key_bounds(c.n_pages, 2, 128)
    A.cache_bounds(dev_cache(A, c), dev(c.pages), dev(c.lens), got)
    x = R.decode(np.stack([codes[:128], codes[126:]]))
    v = values(got)[c.pages[0, 0]]
    assert np.array_equal(v[:, 0], np.floor(2 * x) / 2) and np.array_equal(v[:, 1], np.ceil(2 * x) / 2)


def test_bounds_leave_out_what_has_no_place(A):
    rng = np.random.default_rng(5)
    c = R.make_cache(rng, 4, 2, 64, 64, [200, 100, 64, 90])
    c.pages[0, 1], c.pages[1, 0], c.pages[2, 0] = -1, c.n_pages, 1 << 30
    c.lens = np.array([200, 100, -5, 1 << 30], dtype=np.int32)
    given = np.full((c.n_pages, 2, 2, 64), 2.0)
    got = dev_bounds(given)
    A.cache_bounds(dev_cache(A, c), dev(c.pages), dev(c.lens), got)
    n = c.pages.shape[1] * 64
    c.lens = np.array([200, 100, 0, 1 << 30], dtype=np.int32)
    assert np.array_equal(values(got), P.bounds(c, given, max_q=n))


# ---- choice ----

def choose(A, c, q, G, take, kind="bf16", bnds=None, new=None, check=True, **kw):
    """The lists of the call, equal to those of the definition."""
    cu = None if new is None else cu_of(new)
    max_q = q.shape[0] // len(c.lens) if new is None else max(max(new), 1)
    bnds = P.bounds(c, np.zeros((c.n_pages, c.Hkv, 2, c.d)), max_q=c.pages.shape[1] * c.page) if bnds is None else bnds
    got = A.cache_select(R.torch_q(q, kind).cuda(), dev_cache(A, c), dev(c.pages), dev(c.lens), dev_bounds(bnds), take,
                         cu=None if cu is None else dev(cu), max_q=max_q, **kw).cpu().numpy()
    if check:
        want = P.select(c, q, bnds, G, take, cu=cu, max_q=max_q, **kw)
        bad = np.argwhere((got != want).any(-1))
        assert bad.size == 0, (bad[:3].tolist(), got[tuple(bad[0])].tolist(), want[tuple(bad[0])].tolist())
    return got


def any_queries(rng, T, Hq, d, kind):
    """Queries of the type's whole precision, rows of different sizes."""
    x = rng.standard_normal((T, Hq, d)) * np.exp2(rng.integers(-3, 3, (T, Hq, 1)))
    return R.torch_q(x, kind).double().numpy()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("lens,take", [([1], 1), ([127, 128, 129, 0], 2), ([5000, 31, 700], 5), ([2100, 2048, 2049], 16)])
def test_select_for_single_tokens(A, lens, take, d, page, kind):
    log(f"select {lens} take={take} d={d} page={page} {kind}")
    rng = np.random.default_rng(sum(lens) + d)
    c = R.make_cache(rng, len(lens), 2, page, d, lens)
    choose(A, c, any_queries(rng, len(lens), 8, d, kind), 4, take, kind, n_first=min(1, take - 1), n_last=1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,page,G,run", [(64, 128, 1, 16), (64, 64, 3, 7), (128, 64, 8, 32), (128, 128, 4, 64)])
@pytest.mark.parametrize("lens,new,take", [([40], [40], 1), ([900, 429, 5], [17, 129, 5], 3), ([1500, 0, 1260, 128], [1, 0, 33, 100], 4),
                                           ([3000, 190], [200, 3], 9)])
def test_select_for_runs(A, lens, new, take, d, page, G, run, causal):
    log(f"select {lens} {new} take={take} d={d} page={page} G={G} run={run} causal={causal}")
    rng = np.random.default_rng(sum(lens) + d + G)
    c = R.make_cache(rng, len(lens), 2, page, d, lens)
    q = any_queries(rng, sum(new) + 2, G * 2, d, "bf16")
    choose(A, c, q, G, take, new=new, run=run, causal=causal, n_first=take // 3, n_last=take // 4)


@pytest.mark.parametrize("n,page,take", [(70000, 64, 100), (300000, 64, 1000), (140000, 128, 7), (1 << 20, 64, 16384), (1 << 20, 64, 300)])
def test_select_among_many(A, n, page, take):
    """Up to 16384 pages; all of them one page of the cache but for some."""
    log(f"select among many n={n} page={page} take={take}")
    rng = np.random.default_rng(n)
    c = R.make_cache(rng, 1, 1, page, 64, [page * 40])
    W = n // page
    c.pages = np.concatenate([c.pages, rng.choice(c.pages[0], (1, W - 40))], 1).astype(np.int32)
    c.lens = np.array([n], dtype=np.int32)
    got = choose(A, c, any_queries(rng, 1, 4, 64, "bf16"), 4, take)
    assert (got >= 0).sum() == min(take, W)


@pytest.mark.parametrize("d,G,run", [(64, 2, 1), (128, 8, 3)])
@pytest.mark.parametrize("B,long", [(70, 3000), (140, 400), (140, 2100), (300, 400), (300, 5000), (300, 1500)])
def test_select_of_many_lists(A, B, long, d, G, run):
    """More lists than a split takes: one workgroup a list, of either size, with 16-row and 32-row tiles; a few
    of the sequences are long."""
    log(f"select of many lists B={B} long={long} d={d} G={G} run={run}")
    rng = np.random.default_rng(B + long)
    c = R.make_cache(rng, 1, 1, 64, d, [64 * 50])
    lens = rng.integers(1, 64 * 12, B)
    lens[[0, B // 2]] = 64 * long - 5, 64 * long - 900
    pages = rng.choice(c.pages[0], (B, long)).astype(np.int32)
    c = R.Pages(c.k, c.v, c.ks, c.vs, pages, lens.astype(np.int32))
    new = [int(min(n, run)) for n in lens]
    choose(A, c, any_queries(rng, sum(new), G, d, "bf16"), G, 17, new=new, run=run)


def test_select_takes_the_earlier_of_equals(A):
    rng = np.random.default_rng(8)
    c = R.make_cache(rng, 2, 2, 64, 64, [64 * 30, 64 * 30])
    c.pages[0] = c.pages[0, 3]
    c.pages[1, 5:25] = c.pages[1, 7]
    q = any_queries(rng, 2, 4, 64, "bf16")
    for take in (1, 3, 11, 29, 30, 40):
        got = choose(A, c, q, 2, take, n_first=0, n_last=1)
        m = min(take, 30)
        assert np.array_equal(got[0, 0, 0, :m], [*range(m - 1), 29])
    # as many of them that a histogram does not tell them apart: one workgroup a list, and split
    for W, B in ((700, 1), (700, 300), (3000, 1)):
        c.pages = np.broadcast_to(c.pages[:1, :1], (B, W)).copy()
        c.pages[:, 5::7] = c.pages[0, 0] ^ 1
        c.lens = np.full(B, 64 * W, dtype=np.int32)
        c.lens[1:] = 64 * 3
        choose(A, c, any_queries(rng, B, 4, 64, "bf16"), 2, 131, n_first=0, n_last=1)


def test_select_sums_are_exact(A):
    """Sums next to 2^24 halves: the largest codes and 127s, one channel a half apart."""
    d, page = 128, 64
    c = R.make_cache(np.random.default_rng(9), 1, 1, page, d, [page * 12])
    b = np.zeros((c.n_pages, 1, 2, d))
    c.ks[:] = 127
    for j in range(12):
        b[c.pages[0, j], 0, 1] = 448.0
        b[c.pages[0, j], 0, 1, 5] = 3.5 if j in (4, 9) else 3.0        # 127 a half apart in a sum of 7.2 million
        b[c.pages[0, j], 0, 0] = -448.0
        b[c.pages[0, j], 0, 1, 6] = 1.5 if j == 6 else 1.0
    q = np.full((1, 2, d), 127.0)
    q[0, 0, 6] = 1.0                                                   # one half of the smallest step
    q[0, 1] = 0.0
    choose(A, c, q, 2, 3, bnds=b, n_first=0, n_last=0)
    q[0, 0, 5] = 1.0                                                   # (both channels as small as they get)
    choose(A, c, q, 2, 3, bnds=b, n_first=0, n_last=0)
    q[0, 0] = np.where(np.arange(d) % 2, 127.0, -127.0)
    choose(A, c, q, 2, 5, bnds=b, n_first=0, n_last=0)
    rng = np.random.default_rng(10)
    for _ in range(8):
        lo = R.decode(rng.integers(0, 127, (c.n_pages, 1, d), dtype=np.uint8) | 128)
        hi = R.decode(rng.integers(0, 127, (c.n_pages, 1, d), dtype=np.uint8))
        b = np.stack((np.floor(2 * lo) / 2, np.ceil(2 * hi) / 2), 2)
        q = rng.integers(-127, 128, (1, 2, d)).astype(np.float64)
        q[:, :, 0] = 127
        choose(A, c, q, 2, 4, bnds=b, n_first=0, n_last=0)


def test_select_far_scales_and_queries_that_are_not_finite(A):
    rng = np.random.default_rng(12)
    c = R.make_cache(rng, 3, 2, 64, 64, [64 * 9, 64 * 7 + 5, 64 * 8])
    c.ks = rng.integers(0, 255, c.ks.shape).astype(np.uint8)
    q = any_queries(rng, 3 * 4, 4, 64, "bf16") * np.exp2(rng.integers(-100, 100, (12, 4, 1)).astype(np.float64))
    q = R.torch_q(q, "bf16").double().numpy()
    q[0, 1, 5], q[5, 0, 0], q[5, 1, 63] = np.inf, np.nan, -np.inf
    q[8:] = np.nan                                          # no row of the last sequence takes part
    got = choose(A, c, q, 2, 3, run=2)
    assert np.array_equal(got[2, 0, 0], [0, 1, 7])
    q[:] = 0.0
    choose(A, c, q, 2, 4, run=4)
    q[:] = 2.0 ** -133                                      # bf16's least number
    choose(A, c, q, 2, 4, run=4)


def test_select_pages_that_are_none_and_lengths(A):
    rng = np.random.default_rng(13)
    c = R.make_cache(rng, 4, 2, 64, 64, [600, 300, 200, 640])
    c.pages[0, 2], c.pages[0, 9], c.pages[1, :] = -1, c.n_pages, -3
    q = any_queries(rng, 4, 4, 64, "bf16")
    got = choose(A, c, q, 2, 9)
    assert (got[1] == -1).all()
    choose(A, c, q, 2, 3, max_len=333)
    c.lens = np.array([-3, 1 << 20, 0, 641], dtype=np.int32)
    choose(A, c, q, 2, 3, n_first=0)
    # tokens before position 0 see nothing, those beyond max_q have no list
    c.lens = np.array([5, 40, 70, 300], dtype=np.int32)
    q = any_queries(rng, 40, 4, 64, "bf16")
    choose(A, c, q, 2, 3, new=[10, 10, 10, 10], run=4)


# ---- attention over lists ----

def over_blocks(A, c, q, blocks, G, kind="bf16", new=None, run=1, check=True, out_dtype=torch.float32, max_q=None, **kw):
    T, Hq, d = q.shape
    cu = None if new is None else cu_of(new)
    max_q = (T // len(c.lens) if new is None else max(max(new), 1)) if max_q is None else max_q
    out = torch.full((T, Hq, d), 7.0, dtype=out_dtype, device="cuda")
    lse = torch.full((T, Hq), 7.0, device="cuda")
    A.cache_fwd_blocks(R.torch_q(q, kind).cuda(), dev_cache(A, c), dev(c.pages), dev(c.lens), dev(blocks),
                       cu=None if cu is None else dev(cu), max_q=max_q, run=run, out=out, lse=lse, **kw)
    o, l = out.cpu().double().numpy(), lse.cpu().double().numpy()
    if check:
        compare(o, l, P.attention(c, q, blocks, G, run=run, cu=cu, max_q=max_q, **kw), out_dtype)
    return o, l


def compare(o, l, want, out_dtype):
    w, wl, bound, lb = want
    left = np.isnan(bound)
    assert np.all(o[left] == 7.0) and np.all(l[np.isnan(lb)] == 7.0)
    assert np.array_equal(np.isnan(o[~left]), np.isnan(w[~left]))
    fine = ~left & ~np.isnan(w)
    within(o[fine], w[fine], bound[fine] + (np.abs(w[fine]) * 2.0 ** -8 if out_dtype == torch.bfloat16 else 0.0))
    there = ~np.isnan(lb)
    assert np.array_equal(np.isinf(l[there]), np.isinf(wl[there])) and np.array_equal(np.isnan(l[there]), np.isnan(wl[there]))
    there &= np.isfinite(wl)
    if there.any():
        within(l[there], wl[there], lb[there])


def random_lists(rng, c, runs, take):
    """Blocks in any order, some twice, some none or outside the table."""
    W = c.pages.shape[1]
    x = rng.integers(0, max(-(-int(c.lens.max()) // c.page), 1), (len(c.lens), runs, c.Hkv, take))
    odd = rng.random(x.shape)
    x = np.where(odd < 0.1, -1, np.where(odd < 0.15, W + rng.integers(0, 1 << 30, x.shape), x))
    return np.where((odd > 0.15) & (odd < 0.18), -(1 << 31), x).astype(np.int32)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("lens,take", [([1], 1), ([127, 128, 129, 0], 3), ([2000, 31, 700], 7), ([4000, 65, 3000, 33], 20)])
def test_blocks_for_single_tokens(A, lens, take, d, page, kind):
    log(f"blocks {lens} take={take} d={d} page={page} {kind}")
    rng = np.random.default_rng(len(lens) + d + take)
    c = R.make_cache(rng, len(lens), 2, page, d, lens)
    q = R.make_queries(rng, len(lens), 8, d)
    over_blocks(A, c, q, random_lists(rng, c, 1, take), 4, kind, out_dtype=torch.bfloat16 if take == 7 else torch.float32)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,page,G,run,kind", [(64, 128, 1, 16, "bf16"), (64, 64, 3, 7, "e4m3"), (128, 64, 8, 16, "e4m3"),
                                               (128, 128, 4, 64, "bf16"), (128, 64, 4, 40, "bf16"), (64, 64, 8, 300, "bf16"),
                                               (64, 128, 4, 33, "e4m3"), (128, 128, 4, 32, "e4m3")])
@pytest.mark.parametrize("lens,new,take", [([40], [40], 2), ([900, 429, 5], [17, 129, 5], 4), ([1500, 0, 1260, 128], [1, 0, 33, 100], 6),
                                           ([1000, 290], [200, 3], 9)])
def test_blocks_for_runs(A, lens, new, take, d, page, G, run, kind, causal):
    log(f"blocks {lens} {new} take={take} d={d} page={page} G={G} run={run} {kind} causal={causal}")
    rng = np.random.default_rng(sum(lens) + d + G)
    c = R.make_cache(rng, len(lens), 2, page, d, lens)
    q = R.make_queries(rng, sum(new) + 2, G * 2, d)       # two rows behind the last sequence
    lists = random_lists(rng, c, -(-max(new) // run), take)
    over_blocks(A, c, q, lists, G, kind, new=new, run=run, causal=causal)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("G,take,page,d", [(4, 200, 64, 64), (4, 40, 128, 128), (4, 150, 64, 128), (8, 300, 128, 64)])
@pytest.mark.parametrize("rows", [16, 128])
def test_blocks_in_ranges(A, rows, G, take, page, d, kind):
    """Lists that are split, some of them short, one empty; a loose bound on the tokens of a run makes tall tiles."""
    run = next(r for r in (1, 50, 200, 400, 800, 1600, 3200) if P.blocks_plan(4, G, r, take, page, d, n_cu()).rows == rows)
    plan = P.blocks_plan(4, G, run, take, page, d, n_cu())
    assert plan.rows == rows and plan.ranges > 1
    log(f"blocks in ranges rows={rows} G={G} run={run} take={take} page={page} d={d} {kind} ranges={plan.ranges}")
    rng = np.random.default_rng(take)
    c = R.make_cache(rng, 2, 2, page, d, [1700, 900])
    new = [min(run, 40), min(run, 37)]
    blocks = random_lists(rng, c, 1, take)
    blocks[1, 0, 0] = -1
    blocks[0, 0, 1, 3:] = -1
    over_blocks(A, c, R.make_queries(rng, sum(new), G * 2, d), blocks, G, kind, new=new, run=run, max_q=run)


@pytest.mark.parametrize("d,page,G,run", [(64, 64, 4, 1), (128, 128, 4, 1), (128, 64, 8, 40), (64, 128, 4, 100)])
def test_blocks_all_listed_is_the_whole_cache(A, d, page, G, run):
    rng = np.random.default_rng(21)
    lens = [1000, 130]
    new = [min(run, 100), 1]
    c = R.make_cache(rng, 2, 2, page, d, lens)
    W = c.pages.shape[1]
    blocks = np.broadcast_to(np.arange(W, dtype=np.int32), (2, 1, 2, W))
    q = R.make_queries(rng, sum(new), 2 * G, d)
    o, l = over_blocks(A, c, q, np.ascontiguousarray(blocks), G, new=new, run=run)
    a, b = A.cache_fwd(R.torch_q(q, "bf16").cuda(), dev_cache(A, c), dev(c.pages), dev(c.lens), cu=dev(cu_of(new)), max_q=max(new),
                       out_dtype=torch.float32)
    # FP32 sums of another order, the core's groups of eight as they are
    a, b = a.cpu().double().numpy(), b.cpu().double().numpy()
    within(o, a, 2.0 ** -9 * np.abs(a).max())
    within(l, b, 2.0 ** -17 + 2.0 ** -20 * np.abs(b))


@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 20), (128, 64, 1, 130), (64, 128, 8, 40)])
def test_blocks_nan_values_reach_the_rows_that_see_them(A, d, page, G, new):
    """NaN codes in a listed page: rows before them are as without; in a page that is not listed they reach none."""
    rng = np.random.default_rng(d + new)
    n = 350 + new
    c = R.make_cache(rng, 1, 1, page, d, [n])
    q = R.make_queries(rng, new, G, d)
    t = n - new // 2                                   # a key that the first half of the rows does not see
    pid, slot = int(c.pages[0, t // page]), t % page
    nb = -(-n // page)
    log(f"blocks nan d={d} page={page} G={G} new={new}")
    with_it = np.array([nb - 1, 0, t // page] if t // page < nb - 1 else [t // page, 0, 1], dtype=np.int32).reshape(1, 1, 1, 3)
    without = np.array([0, 1, -1], dtype=np.int32).reshape(1, 1, 1, 3)
    want, wl, bound, lb = P.attention(c, q, with_it, G, run=new)
    ref = over_blocks(A, c, q, without, G, run=new)
    first = t - (n - new)
    c.v[pid, 0, slot, 5] = 0x7F
    c.v[pid, 0, slot, d - 1] = 0xFF
    o, l = over_blocks(A, c, q, with_it, G, run=new, check=False)
    hit = np.zeros(o.shape, dtype=bool)
    hit[first:, :, [5, d - 1]] = True
    assert np.array_equal(np.isnan(o), hit)
    within(np.where(hit, 0, o), np.where(hit, 0, want), bound)
    within(l, wl, lb)
    c.k[pid, 0, slot, 3] = 0x7F
    o, l = over_blocks(A, c, q, with_it, G, run=new, check=False)
    assert np.isnan(o[first:]).all() and np.isnan(l[first:]).all()
    within(o[:first], want[:first], bound[:first])
    within(l[:first], wl[:first], lb[:first])
    o, l = over_blocks(A, c, q, without, G, run=new, check=False)
    assert np.array_equal(o, ref[0]) and np.array_equal(l, ref[1])


@pytest.mark.parametrize("d,page,run", [(64, 64, 1), (128, 128, 1), (128, 64, 64), (64, 128, 64)])
def test_blocks_pages_that_are_none_and_tokens_before_position_0(A, d, page, run):
    rng = np.random.default_rng(23)
    c = R.make_cache(rng, 3, 2, page, d, [500, 300, 200])
    c.pages[0, 1], c.pages[2, 0] = -1, c.n_pages
    c.ks[rng.permutation(c.n_pages)[0]] = 127
    new = [64, 64, 64]
    c.lens = np.array([500, 40, 10], dtype=np.int32)
    lists = random_lists(rng, c, 64 // run, 4)
    o, l = over_blocks(A, c, R.make_queries(rng, 192, 8, d), lists, 4, new=new, run=run)
    assert np.isinf(l[64:88]).all() and (o[64:88] == 0).all()


def test_blocks_queries_with_strides_and_descales(A):
    rng = np.random.default_rng(24)
    c = R.make_cache(rng, 2, 2, 64, 64, [300, 200])
    q = R.make_queries(rng, 2, 8, 64)
    wide = torch.zeros((2, 12, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:10] = R.torch_q(q, "bf16").cuda()
    lists = random_lists(rng, c, 1, 4)
    out, lse = A.cache_fwd_blocks(wide[:, 2:10], dev_cache(A, c), dev(c.pages), dev(c.lens), dev(lists), sm_scale=0.3, q_descale=0.5,
                                  out_dtype=torch.float32)
    want = P.attention(c, q, lists, 4, sm_scale=0.3, q_descale=0.5)
    compare(out.cpu().double().numpy(), lse.cpu().double().numpy(), want, torch.float32)
    none = A.cache_fwd_blocks(wide[:, 2:10], dev_cache(A, c), dev(c.pages), dev(c.lens), dev(lists), sm_scale=0.3, q_descale=0.5,
                              out_dtype=torch.float32, want_lse=False)
    assert none[1] is None and torch.equal(none[0], out)


# ---- a shared prefix ----

def over_shared(A, c, q, n_shared, G, kind="bf16", new=None, check=True, out_dtype=torch.float32, max_q=None, max_len=0, **kw):
    T, Hq, d = q.shape
    cu = None if new is None else cu_of(new)
    max_q = (T // len(c.lens) if new is None else max(max(new), 1)) if max_q is None else max_q
    out = torch.full((T, Hq, d), 7.0, dtype=out_dtype, device="cuda")
    lse = torch.full((T, Hq), 7.0, device="cuda")
    pages = c.pages.copy()
    if n_shared < pages.shape[1]:
        pages[1:, :n_shared] = -9                          # not looked at
    A.cache_fwd_shared(R.torch_q(q, kind).cuda(), dev_cache(A, c), dev(pages), dev(c.lens), n_shared,
                       cu=None if cu is None else dev(cu), max_q=max_q, out=out, lse=lse, max_len=max_len, **kw)
    o, l = out.cpu().double().numpy(), lse.cpu().double().numpy()
    if check:
        compare(o, l, P.attention(c, q, None, G, run=max_q, cu=cu, max_q=max_q, **kw), out_dtype)
    return o, l


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("lens,shared", [([130], 1), ([300, 257, 256, 10, 0], 2), ([900] + [770 + i for i in range(9)], 6),
                                         ([600, 400], 0), ([640, 640, 640], 5)])
def test_shared_for_single_tokens(A, lens, shared, d, page, kind):
    log(f"shared {lens} {shared} d={d} page={page} {kind}")
    rng = np.random.default_rng(len(lens) + d + shared)
    c = P.share(R.make_cache(rng, len(lens), 2, page, d, lens), shared)
    over_shared(A, c, R.make_queries(rng, len(lens), 8, d), shared, 4, kind,
                out_dtype=torch.bfloat16 if shared == 2 else torch.float32)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,page,G,kind", [(64, 128, 1, "bf16"), (64, 64, 3, "e4m3"), (128, 64, 8, "e4m3"), (128, 128, 4, "bf16")])
@pytest.mark.parametrize("lens,new,shared", [([300], [40], 2), ([900, 829, 805], [17, 129, 5], 6), ([500, 0, 400, 128], [1, 0, 33, 100], 3),
                                             ([700, 690], [200, 3], 4), ([400, 380, 200], [150, 140, 200], 2)])
def test_shared_for_chunks(A, lens, new, shared, d, page, G, kind, causal):
    """The last two: tokens whose own keys lie among the shared pages, a sequence that ends in them."""
    log(f"shared {lens} {new} {shared} d={d} page={page} G={G} {kind} causal={causal}")
    rng = np.random.default_rng(sum(lens) + d + G)
    c = P.share(R.make_cache(rng, len(lens), 2, page, d, lens), shared)
    q = R.make_queries(rng, sum(new) + 2, G * 2, d)       # two rows behind the last sequence
    over_shared(A, c, q, shared, G, kind, new=new, causal=causal)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("G,shared,n,page,d", [(4, 20, 2700, 128, 128), (4, 40, 2700, 64, 64), (8, 10, 1500, 128, 64), (8, 21, 1500, 64, 128),
                                               (2, 300, 40000, 128, 64), (2, 300, 20000, 64, 128), (1, 40, 6000, 64, 128), (4, 120, 17000, 128, 128)])
@pytest.mark.parametrize("pre_rows,own_rows", [(16, 16), (128, 16), (16, 128), (128, 128)])
def test_shared_on_each_kernel(A, pre_rows, own_rows, G, shared, n, page, d, kind):
    """Loose bounds on the tokens (of the call, of a sequence) make tall tiles."""
    B, W, base = 4, -(-n // page), shared * page
    found = [(t, m) for t in (4, 30, 300, 600, 1000, 2000, 4000, 8000) for m in (1, 9, 100, 200, 400, 800, 1600) if t == 4 or m > 1
             for p in [P.shared_plan(B, 2, G, t, m, shared, W * page, page, d, n_cu())] if (p.pre.rows, p.own.rows) == (pre_rows, own_rows)]
    if not found:
        assert (pre_rows, own_rows, d) == (16, 16, 128)     # (128-row tiles are faster there)
        pytest.skip("no call of these sizes takes these tiles")
    T, max_q = found[0]
    plan = P.shared_plan(B, 2, G, T, max_q, shared, W * page, page, d, n_cu())
    log(f"shared rows {pre_rows} {own_rows} G={G} shared={shared} n={n} page={page} d={d} {kind} T={T} max_q={max_q} ranges {plan.pre.ranges} {plan.own.ranges}")
    rng = np.random.default_rng(n + d)
    c = R.make_cache(rng, 1, 2, page, d, [n], extra=B * (W - shared) + 2)
    c.k[c.k & 127 == 127], c.v[c.v & 127 == 127] = 0x30, 0x31
    spare = np.array([p for p in range(c.n_pages) if p not in c.pages[0]])[:(B - 1) * (W - shared)].reshape(B - 1, -1)
    pages = np.concatenate([c.pages, np.concatenate([c.pages[[0] * (B - 1), :shared], spare], 1)]).astype(np.int32)
    lens = [n, *(int(x) for x in rng.integers(base + 1, n, B - 1))]
    c = R.Pages(c.k, c.v, c.ks, c.vs, pages, np.array(lens, dtype=np.int32))
    new = [9, 8, 1, 7] if T > 4 else [1, 1, 1, 1]
    over_shared(A, c, R.make_queries(rng, T, 2 * G, d), shared, G, kind, new=new, max_q=max_q)


@pytest.mark.parametrize("B,G,new", [(5, 4, 1), (3, 8, 40), (40, 4, 1)])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 128)])
def test_shared_pages_that_are_none_and_lengths(A, d, page, B, G, new):
    rng = np.random.default_rng(31)
    c = P.share(R.make_cache(rng, B, 2, page, d, [700] * B), 4)
    c.pages[:, 2], c.pages[0, 5] = -1, c.n_pages
    c.lens = rng.integers(-20, 900, B).astype(np.int32)
    q = R.make_queries(rng, B * new, 2 * G, d)
    over_shared(A, c, q, 4, G)
    # a bound inside and before the shared pages' end
    for max_len in (4 * page + 70, 4 * page, 2 * page + 9, 1):
        cut = R.Pages(c.k, c.v, c.ks, c.vs, c.pages, c.lens)
        o, l = over_shared(A, c, q, 4, G, max_len=max_len, check=False)
        a, b = A.cache_fwd(R.torch_q(q, "bf16").cuda(), dev_cache(A, cut), dev(c.pages), dev(c.lens), max_len=max_len, out_dtype=torch.float32)
        a, b = a.cpu().double().numpy(), b.cpu().double().numpy()
        assert np.array_equal(np.isnan(o), np.isnan(a)) and np.array_equal(np.isnan(l), np.isnan(b)) and np.array_equal(np.isinf(l), np.isinf(b))
        top = np.abs(np.nan_to_num(a)).max()
        within(np.nan_to_num(o), np.nan_to_num(a), 2.0 ** -9 * max(top, 1e-30))
        fine = np.isfinite(b)
        within(l[fine], b[fine], 2.0 ** -17 + 2.0 ** -20 * np.abs(b[fine])) if fine.any() else None


@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 20), (128, 64, 1, 60), (64, 128, 8, 40)])
def test_shared_nan_values_reach_the_rows_that_see_them(A, d, page, G, new):
    """A NaN in a shared page reaches the sequences whose tokens see it; the second ends before it."""
    rng = np.random.default_rng(d + new)
    base = 3 * page
    lens = [base + new + 9, base - 20, base + 2 * new]
    c = P.share(R.make_cache(rng, 3, 1, page, d, lens), 3)
    q = R.make_queries(rng, 3 * new, G, d)
    log(f"shared nan d={d} page={page} G={G} new={new}")
    want, wl, bound, lb = R.attention(c, q, G)
    pid = int(c.pages[0, 2])
    c.v[pid, 0, page - 3, 5] = 0x7F
    c.v[pid, 0, page - 3, d - 1] = 0xFF
    o, l = over_shared(A, c, q, 3, G, check=False)
    hit = np.zeros(o.shape, dtype=bool)
    for rows in (slice(0, new), slice(2 * new, 3 * new)):
        hit[rows][:, :, [5, d - 1]] = True
    assert np.array_equal(np.isnan(o), hit)
    within(np.where(hit, 0, o), np.where(hit, 0, want), bound)
    within(l, wl, lb)
    c.k[pid, 0, page - 3, 3] = 0x7F
    o, l = over_shared(A, c, q, 3, G, check=False)
    assert np.isnan(o[:new]).all() and np.isnan(l[2 * new:]).all()
    within(o[new:2 * new], want[new:2 * new], bound[new:2 * new])


def test_shared_far_scales_and_values(A):
    """Blocks of far apart scales on both sides of the prefix's end, a far maximum in either."""
    for seed in range(6):
        rng = np.random.default_rng(40 + seed)
        B = 2 if seed % 2 else 40
        c = P.share(R.make_cache(rng, B, 2, 64, 64, [640] * B, spread=6), 5)
        far = c.pages[0, 2] if seed % 3 else c.pages[0, 7]
        c.ks[far] = 131
        c.vs[c.pages[0, 3]] = 127 + (80 if seed < 3 else -80)
        over_shared(A, c, R.make_queries(rng, B, 8, 64), 5, 4)


# ---- a run of the operators, graphs, streams ----

def step(A, cache, pages, lens, qkv, Hq, Hkv, bounds, table, take, max_q=1, run=1, cu=None, **kw):
    """Append, bounds, choice and attention of one step, as a program makes them."""
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    q = A.cache_append(cache, k, v, pages, lens, table=table, q=q, max_q=max_q, cu=cu, **kw)
    A.cache_bounds(cache, pages, lens, bounds, max_q=max_q, cu=cu, **kw)
    lists = A.cache_select(q, cache, pages, lens, bounds, take, max_q=max_q, run=run, cu=cu, **kw)
    out, lse = A.cache_fwd_blocks(q, cache, pages, lens, lists, max_q=max_q, run=run, cu=cu, out_dtype=torch.float32, **kw)
    return q, lists, out, lse


def as_pages(c, gc, lens):
    """The GPU's cache as a reference's."""
    k, v, ks, vs = (t.view(torch.uint8).cpu().numpy() for t in gc)
    return R.Pages(k, v, ks, vs, c.pages, np.array(lens, dtype=np.int32))


@pytest.mark.parametrize("d,page", [(64, 64), (128, 128)])
def test_prompt_then_tokens_behind_a_shared_prefix(A, d, page):
    """Three requests behind a common prompt: the prompt is written once, a ragged chunk of each follows, then
    single tokens on lists and, beside them, on all keys by the shared call; every step against 64 bits."""
    rng = np.random.default_rng(61)
    B, Hq, Hkv, G, base = 3, 8, 2, 4, 3
    c = R.make_cache(rng, B, Hkv, page, d, [12 * page] * B, extra=0)
    c.pages[1:, :base] = c.pages[0, :base]
    pages, table, gc = dev(c.pages), A.rope_table(12 * page, d), dev_cache(A, c)
    bounds = A.key_bounds(c.n_pages, Hkv, d)
    # the prompt, as one sequence
    n = base * page
    x = torch.randn((n, Hq + 2 * Hkv, d), device="cuda").bfloat16()
    one = torch.tensor([n], dtype=torch.int32, device="cuda")
    step(A, gc, pages[:1].contiguous(), one, x, Hq, Hkv, bounds, table, 2, max_q=n, run=n)
    lens, new = np.array([n, n, n]), [70, 1, 33]
    for i in range(4):
        lens = lens + new
        cu = dev(cu_of(new)) if max(new) > 1 else None
        x = torch.randn((sum(new), Hq + 2 * Hkv, d), device="cuda").bfloat16()
        log(f"step {i} lens {lens.tolist()}")
        run = 16 if max(new) > 1 else 1
        q, lists, out, lse = step(A, gc, pages, dev(lens.astype(np.int32)), x, Hq, Hkv, bounds, table, 3, max_q=max(new), run=run, cu=cu)
        now = as_pages(c, gc, lens)
        qs = q.double().cpu().numpy()
        # the pages' bounds are those of all their tokens, the lists those of the definition
        want = P.bounds(now, values(bounds), max_q=12 * page)
        assert np.array_equal(values(bounds), want)
        assert np.array_equal(lists.cpu().numpy(), P.select(now, qs, want, G, 3, run=run, cu=cu_of(new), max_q=max(new)))
        kw = dict(cu=cu_of(new), max_q=max(new))
        compare(out.double().cpu().numpy(), lse.double().cpu().numpy(), P.attention(now, qs, lists.cpu().numpy(), G, run=run, **kw), torch.float32)
        out, lse = A.cache_fwd_shared(q, gc, pages, dev(lens.astype(np.int32)), base, cu=cu, max_q=max(new), out_dtype=torch.float32)
        compare(out.double().cpu().numpy(), lse.double().cpu().numpy(), P.attention(now, qs, None, G, **kw), torch.float32)
        new = [1, 1, 1]


@pytest.mark.parametrize("d,page,B", [(64, 64, 3), (128, 128, 3), (128, 64, 20)])
def test_captured_step_follows_the_lengths(A, d, page, B):
    """The step captured once, replayed while the lengths grow, beside eager calls: equal to eager steps; with it the
    call behind a shared prefix."""
    rng = np.random.default_rng(62)
    Hq, Hkv, base, W = 8, 2, 4, 40
    c = R.make_cache(rng, B, Hkv, page, d, [W * page] * B)
    c.pages[1:, :base] = c.pages[0, :base]
    start = (base * page + rng.integers(1, 30 * page, B)).astype(np.int32)
    table, pages = A.rope_table(W * page, d), dev(c.pages)
    xs = [torch.randn((B, Hq + 2 * Hkv, d), device="cuda").bfloat16() for _ in range(4)]

    def both(cache, bounds, lens, x):
        r = step(A, cache, pages, lens, x, Hq, Hkv, bounds, table, 9)
        return (*r, *A.cache_fwd_shared(r[0], cache, pages, lens, base))

    def fresh():
        gc, b = dev_cache(A, c), A.key_bounds(c.n_pages, Hkv, d)
        A.cache_bounds(gc, pages, dev(start), b)
        return gc, b

    ge, be = fresh()
    eager = []
    for i, x in enumerate(xs):
        eager.append([t.clone() for t in both(ge, be, dev(start + 1 + i), x)])
    gg, bg = fresh()
    lens, x = dev(start + 1), xs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(*fresh(), lens, x)                                 # warm
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(gg, bg, lens, x)
    for i, xi in enumerate(xs):
        log(f"replay {i}")
        x.copy_(xi)
        lens.copy_(dev(start + 1 + i))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, eager[i]):
            assert torch.equal(a, b)
        both(ge, be, lens, x)                                   # eager work between


def test_calls_on_another_stream_and_two_at_once(A):
    """Each call behind late inputs on a stream of its own; split calls, each with a workspace of its own, side by
    side on two streams and in two graphs that are replayed in turn."""
    rng = np.random.default_rng(63)
    sets = []
    for n in (9000, 20000):
        c = R.make_cache(rng, 2, 2, 64, 128, [n, 1000])
        c.pages[1, :10] = c.pages[0, :10]
        b = dev_bounds(P.bounds(c, np.zeros((c.n_pages, 2, 2, 128)), max_q=1 << 20))
        q = R.torch_q(R.make_queries(rng, 2, 8, 128), "bf16").cuda()
        args = (dev_cache(A, c), dev(c.pages), dev(c.lens))
        W = c.pages.shape[1]
        shape = (A.attn_fp8_cache(None, None, None, None, c.n_pages, 2, 64, 128), A.attn_fp8_batch(None, None, None, 2, W, 2, 1))
        assert A.attn_fp8_cache_blocks_workspace_bytes(*shape, 8, 60, 1)[1] > 0 and A.attn_fp8_cache_shared_workspace_bytes(*shape, 10, 8, 0)[1] > 0
        assert n < 17000 or A.attn_fp8_cache_select_workspace_bytes(*shape, 8, 60, 1, 0)[1] > 0

        def calls(q, args=args, b=b, **kw):
            lists = A.cache_select(q, *args, b, 60, **kw)
            return [lists, *A.cache_fwd_blocks(q, *args, lists, **kw), *A.cache_fwd_shared(q, *args, 10, **kw)]
        sets.append((calls, q, calls(q)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for (calls, q, _), s in zip(sets, streams):
        late = torch.zeros_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)
            late.copy_(q)
        got.append([calls(late, stream=s) for _ in range(6)])
    torch.cuda.synchronize()
    for (_, _, want), runs in zip(sets, got):
        for r in runs:
            assert all(torch.equal(a, b) for a, b in zip(r, want))
    graphs = []
    for calls, q, want in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = calls(q)
        graphs.append((g, r, want))
    for i in range(4):
        log(f"replay {i}")
        for g, r, want in graphs:
            r[1].fill_(3.0)
            g.replay()
        sets[0][0](sets[0][1])
        torch.cuda.synchronize()
        for _, r, want in graphs:
            assert all(torch.equal(a, b) for a, b in zip(r, want))


def test_cache_beyond_four_gigabytes(A):
    """Pages whose offsets pass 32 bits, read by every call."""
    page, d, Hkv, n_pages = 128, 128, 8, 70000                  # 9.2 GB of K
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    k = torch.zeros((n_pages, Hkv, page, d), dtype=torch.uint8, device="cuda")
    v, s = torch.zeros_like(k), torch.full((n_pages, Hkv), 127, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(64)
    ids = np.array([[69999, 3, 40000, 69000, 33333, 50001]], dtype=np.int32)
    small = R.make_cache(rng, 1, Hkv, page, d, [6 * page - 5], extra=0)
    order = small.pages[0]
    for j, p in enumerate(ids[0]):
        k[int(p)], v[int(p)] = dev(small.k[order[j]]), dev(small.v[order[j]])
        s[int(p)] = dev(small.ks[order[j]])
    vs = s.clone()
    for j, p in enumerate(ids[0]):
        vs[int(p)] = dev(small.vs[order[j]])
    gc = A.KVCache(k.view(E4M3), v.view(E4M3), s, vs)
    bounds = A.key_bounds(n_pages, Hkv, d)
    pages, lens = dev(ids), dev(small.lens)
    q = R.make_queries(rng, 1, 16, d)
    gq = R.torch_q(q, "bf16").cuda()
    A.cache_bounds(gc, pages, lens, bounds)
    want = P.bounds(small, np.zeros((small.n_pages, Hkv, 2, d)), max_q=6 * page)
    assert np.array_equal(values(bounds[torch.from_numpy(ids[0]).long().cuda()]), want[order])
    lists = A.cache_select(gq, gc, pages, lens, bounds, 3)
    assert np.array_equal(lists.cpu().numpy(), P.select(small, q, want, 2, 3))
    out, lse = A.cache_fwd_blocks(gq, gc, pages, lens, lists, out_dtype=torch.float32)
    compare(out.cpu().double().numpy(), lse.cpu().double().numpy(), P.attention(small, q, lists.cpu().numpy(), 2), torch.float32)
    out, lse = A.cache_fwd_shared(gq, gc, pages, lens, 4, out_dtype=torch.float32)
    compare(out.cpu().double().numpy(), lse.cpu().double().numpy(), P.attention(small, q, None, 2), torch.float32)


def test_offsets_outside_the_call(A):
    """Entries of cu outside 0 .. T, out of order or past max_q: nothing but the rows in place is written."""
    rng = np.random.default_rng(65)
    c = P.share(R.make_cache(rng, 4, 2, 64, 64, [300, 290, 280, 270]), 2)
    q = R.make_queries(rng, 20, 4, 64)
    gq, args = R.torch_q(q, "bf16").cuda(), (dev_cache(A, c), dev(c.pages), dev(c.lens))
    bounds = P.bounds(c, np.zeros((c.n_pages, 2, 2, 64)), max_q=320)
    for cu in ([-5, 3, 3, 9, 100], [4, 4, 2, 2, 8], [0, 1 << 30, -(1 << 31), 5, 6]):
        gcu = dev(np.array(cu, dtype=np.int32))
        lists = A.cache_select(gq, *args, dev_bounds(bounds), 3, cu=gcu, max_q=5, run=2)
        assert lists.shape == (4, 3, 2, 3) and int(lists.min()) >= -1 and int(lists.max()) < 5
        out = torch.full((20, 4, 64), 7.0, device="cuda")
        o1, _ = A.cache_fwd_blocks(gq, *args, lists, cu=gcu, max_q=5, run=2, out=out)
        o2, _ = A.cache_fwd_shared(gq, *args, 2, cu=gcu, max_q=5, out=torch.full_like(out, 7.0))
        o3, _ = A.cache_fwd(gq, *args, cu=gcu, max_q=5, out=torch.full_like(out, 7.0))
        written = lambda o: (o != 7.0).any(-1).any(-1)
        assert torch.equal(written(o1), written(o3)) and torch.equal(written(o2), written(o3))
        A.cache_bounds(*args, dev_bounds(bounds), cu=gcu, max_q=5)


def test_binding_refuses_what_does_not_fit(A):
    c = R.make_cache(np.random.default_rng(66), 2, 2, 64, 64, [300, 200])
    gc, pages, lens = dev_cache(A, c), dev(c.pages), dev(c.lens)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    b, lists = A.key_bounds(c.n_pages, 2, 64), torch.zeros((2, 1, 2, 3), dtype=torch.int32, device="cuda")
    bad = [
        lambda: A.cache_bounds(gc, pages, lens, b[:1]),
        lambda: A.cache_bounds(gc, pages, lens, b.float()),
        lambda: A.cache_bounds(gc, pages, lens, b.transpose(1, 2)),
        lambda: A.cache_bounds(gc, pages, lens[:1], b),
        lambda: A.cache_bounds(gc, pages, lens, b, max_q=-1),
        lambda: A.cache_bounds(gc, pages, lens, b, cu=lens),
        lambda: A.cache_select(q, gc, pages, lens, b, 0),
        lambda: A.cache_select(q, gc, pages, lens, b, 3, run=0),
        lambda: A.cache_select(q, gc, pages, lens, b.cpu(), 3),
        lambda: A.cache_select(q, gc, pages, lens, b, 3, blocks=lists[..., :2]),
        lambda: A.cache_select(q[:, :3], gc, pages, lens, b, 3),
        lambda: A.cache_select(q.float(), gc, pages, lens, b, 3),
        lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists.long()),
        lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists[:1]),
        lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists[0]),
        lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists.transpose(1, 2)),
        lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists, max_q=2),
        lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists, run=0),
        lambda: A.cache_fwd_blocks(q.half(), gc, pages, lens, lists),
        lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists, out=torch.zeros((2, 4, 32), device="cuda")),
        lambda: A.cache_fwd_shared(q, gc, pages, lens, 1, lse=torch.zeros((2, 3), device="cuda")),
        lambda: A.cache_fwd_shared(q, gc, pages, lens, 1 << 40),
        lambda: A.cache_fwd_shared(q, gc, pages.cpu(), lens, 1),
    ]
    for i, f in enumerate(bad):
        log(f"refusal {i}")
        with pytest.raises((ValueError, TypeError)):
            f()
    for f in (lambda: A.cache_select(q, gc, pages, lens, b, 3, n_first=2, n_last=2), lambda: A.cache_select(q, gc, pages, lens, b, 3, n_first=-1),
              lambda: A.cache_select(q, gc, pages, lens, b, 1 << 20), lambda: A.cache_fwd_shared(q, gc, pages, lens, 6),
              lambda: A.cache_fwd_shared(q, gc, pages, lens, -1), lambda: A.cache_fwd_blocks(q, gc, pages, lens, lists[..., :0].contiguous())):
        with pytest.raises(A.AttnError):
            f()


def test_calls_without_tokens(A):
    c = R.make_cache(np.random.default_rng(67), 2, 2, 64, 64, [300, 200])
    gc, pages, lens = dev_cache(A, c), dev(c.pages), dev(c.lens)
    b = A.key_bounds(c.n_pages, 2, 64)
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    lists = A.cache_select(q, gc, pages, lens, b, 3, blocks=torch.full((2, 1, 2, 3), 9, dtype=torch.int32, device="cuda"))
    assert (lists == -1).all()
    assert A.cache_fwd_blocks(q, gc, pages, lens, lists)[0].shape == (0, 4, 64)
    assert A.cache_fwd_shared(q, gc, pages, lens, 1)[0].shape == (0, 4, 64)
    none = (gc, pages[:0].contiguous(), lens[:0].contiguous())
    assert A.cache_select(q, *none, b, 3).shape == (0, 1, 2, 3)
    assert A.cache_fwd_shared(q, *none, 1)[0].shape == (0, 4, 64)
    A.cache_bounds(*none, b)
    A.cache_bounds(gc, pages, lens, b, max_q=0)
    assert (values(b) == 0).all()
    # an empty page table
    narrow = (gc, pages[:, :0].contiguous(), lens)
    one = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert (A.cache_select(one, *narrow, b, 3) == -1).all()
    for o, l in (A.cache_fwd_blocks(one, *narrow, lists), A.cache_fwd_shared(one, *narrow, 0)):
        assert (o == 0).all() and torch.isinf(l).all()


@pytest.mark.parametrize("page", [64, 128])
def test_calls_of_no_sequences_with_wide_tables(A, page):
    """Tables of more pages than one workgroup's waves choose among, of no sequence."""
    c = A.kv_cache(3, 2, 64, page=page)
    b = A.key_bounds(3, 2, 64)
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    lens = torch.zeros((0,), dtype=torch.int32, device="cuda")
    for W in (257, 600, 16384):
        log(f"no sequences page={page} W={W}")
        pages = torch.zeros((0, W), dtype=torch.int32, device="cuda")
        lists = A.cache_select(q, c, pages, lens, b, 3)
        assert lists.shape == (0, 1, 2, 3)
        assert A.cache_fwd_blocks(q, c, pages, lens, lists)[0].shape == (0, 4, 64)
        assert A.cache_fwd_shared(q, c, pages, lens, 2)[0].shape == (0, 4, 64)
        assert A.cache_bounds(c, pages, lens, b) is b
        # sequences without new tokens beside it: empty lists
        some = torch.zeros((2, W), dtype=torch.int32, device="cuda")
        lists = A.cache_select(q, c, some, torch.full((2,), W * page, dtype=torch.int32, device="cuda"), b, 3,
                               blocks=torch.full((2, 1, 2, 3), 9, dtype=torch.int32, device="cuda"))
        assert (lists == -1).all()


@pytest.mark.parametrize("B,W,Hkv,page", [(3, 1 << 20, 16, 64), (3, 400000, 16, 128), (300, 40000, 1, 128), (300, 100000, 1, 128), (700, 30000, 8, 64)])
def test_bounds_of_all_tokens_with_wide_tables(A, B, W, Hkv, page):
    """max_q=None on tables with room for far more tokens than there are, more than a batch may have (2^30) and than
    a launch has workgroups for (2^24): the bounds are those of the tokens there are."""
    log(f"bounds of wide tables B={B} W={W} Hkv={Hkv} page={page}")
    rng = np.random.default_rng(B)
    c = R.make_cache(rng, 4, Hkv, page, 64, [700, 130, 1, 1000])
    wide = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
    lens = np.zeros(B, dtype=np.int32)
    at = [0, B // 2, B - 1]
    for b, i in zip(at, range(3)):
        wide[b, :c.pages.shape[1]] = dev(c.pages[i])
        lens[b] = c.lens[i]
    given = np.full((c.n_pages, Hkv, 2, 64), 1.5)
    got = dev_bounds(given)
    A.cache_bounds(dev_cache(A, c), wide, dev(lens), got)
    few = R.Pages(c.k, c.v, c.ks, c.vs, c.pages[:3], c.lens[:3])
    assert np.array_equal(values(got), P.bounds(few, given, max_q=W * page))
    # a sequence that fills its table
    last = torch.full((1, W), int(c.pages[3, 0]), dtype=torch.int32, device="cuda")
    last[0, W - c.pages.shape[1]:] = dev(c.pages[3])
    got = dev_bounds(given)
    A.cache_bounds(dev_cache(A, c), last, dev(np.array([W * page], dtype=np.int32)), got)
    full = R.Pages(c.k, c.v, c.ks, c.vs, c.pages[3:], np.array([c.pages.shape[1] * page], dtype=np.int32))
    assert np.array_equal(values(got), P.bounds(full, given, max_q=W * page))


# Table widths and lengths of a choice's four forms, by the number of its lists and the pages there may be:
# parts of a list by workgroups of their own (few lists of many pages), a workgroup a list for up to 16384 pages,
# for up to 2048 of many lists (four waves) and of few (eight).
FORMS = {"split": (2, 700), "large": (140, 2100), "many": (300, 400), "few": (140, 300)}


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,run", [(4, 3), (3, 11), (8, 40)])
@pytest.mark.parametrize("form", FORMS)
def test_select_in_each_form(A, form, G, run, d, kind):
    """Every kernel of the choice: 16-row tiles (run * G up to 16), 32-row tiles of fewer and of more tiles than waves."""
    B, W = FORMS[form]
    rng = np.random.default_rng(B + G + d)
    heads = 2 if form == "split" else 1
    c = R.make_cache(rng, 1, heads, 64, d, [64 * 40])
    lens = rng.integers(1, 64 * 9, B)
    lens[0], lens[B // 2] = 64 * W - 5, 64 * W * 3 // 4
    pages = rng.choice(c.pages[0], (B, W)).astype(np.int32)
    c = R.Pages(c.k, c.v, c.ks, c.vs, pages, lens.astype(np.int32))
    new = [int(min(n, 1 + i % run)) for i, n in enumerate(lens)]
    new[0] = new[B // 2] = run
    size = A.attn_fp8_cache_select_workspace_bytes(A.attn_fp8_cache(None, None, None, None, c.n_pages, heads, 64, d),
                                                   A.attn_fp8_batch(None, None, None, B, W, sum(new), run), heads * G, 17, run, 0)
    assert size == (0, 4 * B * heads * W if form == "split" else 0) and (W > 2048) == (form == "large") and (B > 256) == (form == "many")
    log(f"select form={form} G={G} run={run} d={d} {kind}")
    choose(A, c, any_queries(rng, sum(new), G * heads, d, kind), G, 17, kind, new=new, run=run)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page,n,take", [(128, 64, 131001, 128), (64, 64, 1 << 20, 300), (128, 128, 1 << 21, 16384)])
def test_select_for_one_long_request(A, d, page, n, take, kind):
    """Up to 16384 pages of one sequence, single tokens of four heads: parts of the list by several workgroups."""
    rng = np.random.default_rng(n)
    c = R.make_cache(rng, 1, 1, page, d, [page * 40])
    W = -(-n // page)
    c.pages = np.concatenate([c.pages, rng.choice(c.pages[0], (1, W - 40))], 1).astype(np.int32)
    c.lens = np.array([n], dtype=np.int32)
    log(f"select one long request n={n} page={page} d={d} take={take} {kind}")
    got = choose(A, c, any_queries(rng, 1, 4, d, kind), 4, take, kind)
    assert (got >= 0).sum() == min(take, W)


@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("run", [1, 2, 16, 64, 65, 100, 128, 129, 200])
def test_tokens_of_a_run_keep_their_own_pages(A, run, page):
    """n_last = 1 + ceil((run - 1) / page): a run that crosses the ends of pages has the pages of all of its tokens, so
    every token sees itself."""
    rng = np.random.default_rng(run)
    lens, new = [900, 517, 64, 300], [400, 129, 64, 7]
    c = R.make_cache(rng, 4, 1, page, 64, lens)
    q = any_queries(rng, sum(new), 2, 64, "bf16")
    n_last = 1 + -(-(run - 1) // page)
    log(f"select keeps own pages run={run} page={page}")
    got = choose(A, c, q, 2, n_last, new=new, run=run, n_first=0, n_last=n_last)
    for b in range(4):
        for i in range(new[b]):
            assert (lens[b] - new[b] + i) // page in got[b, i // run, 0]
    out, lse = over_blocks(A, c, q, got, 2, new=new, run=run)
    assert np.isfinite(lse).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("pre_rows", [16, 128])
def test_shared_rows_of_no_sequence_take_no_part(A, pre_rows, d, page, kind):
    """Rows of q behind the last sequence, and shared pages that lie behind all of them, may hold anything: the
    result is the same to the last bit."""
    rng = np.random.default_rng(71 + d + page)
    shared, W, G = 7, 9, 4
    lens, new = [5 * page - 3, 4 * page + 9, 4 * page + 30], [9, 1, 7]
    c = P.share(R.make_cache(rng, 3, 2, page, d, [W * page] * 3), shared)
    c.lens = np.array(lens, dtype=np.int32)
    T = next(t for t in (40, 300, 600, 1000, 2000, 4000, 8000, 16000)
             if P.shared_plan(3, 2, G, t, 9, shared, W * page, page, d, n_cu()).pre.rows == pre_rows)
    q = np.zeros((T, 2 * G, d))
    q[:sum(new)] = R.make_queries(rng, sum(new), 2 * G, d)
    log(f"shared rows of no sequence rows={pre_rows} T={T} d={d} page={page} {kind}")
    want = over_shared(A, c, q, shared, G, kind, new=new)
    for pad in (math.inf, math.nan, 448.0):
        x = q.copy()
        x[sum(new):, ::2] = pad
        got = over_shared(A, c, x, shared, G, kind, new=new, check=False)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]), pad
    x = q.copy()
    x[sum(new):] = 400.0
    for p in c.pages[0, 5:shared]:
        c.k[p], c.v[p], c.ks[p], c.vs[p] = 0x7E, 0x7F, 254, 255
    got = over_shared(A, c, x, shared, G, kind, new=new, check=False)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_select_refuses_sizes_before_it_allocates(A):
    """A list of more pages than the call takes is refused by its size, not by the memory that it would need."""
    c = A.kv_cache(3, 8, 64, page=64)
    pages = torch.zeros((64, 4), dtype=torch.int32, device="cuda")
    lens = torch.full((64,), 200, dtype=torch.int32, device="cuda")
    q = torch.zeros((64, 8, 64), dtype=torch.bfloat16, device="cuda")
    b = A.key_bounds(3, 8, 64)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.max_memory_allocated()
    for take in (16385, 1 << 18, (1 << 31) - 1):
        log(f"refused take={take}")
        with pytest.raises(A.AttnError):
            A.cache_select(q, c, pages, lens, b, take)
    assert torch.cuda.max_memory_allocated() == before
