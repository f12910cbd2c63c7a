"""The cache attention on tiles of 128 query rows, and its splits: every case names the kernel it
runs, by the library's own plan.  A bound on the new tokens above what a batch has puts small
batches on those tiles, so that the 64-bit results stay cheap."""
import math

import numpy as np
import pytest
import torch

from tests import cache_ref as R
from tests.cache_plan import fwd_plan, max_q_of_tall_tiles
from tests.gpu_helpers import log
from tests.test_gpu_cache import cu_of, dev, dev_cache, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2606_06521_amd import attn_fp8
    return attn_fp8


def n_cu():
    return torch.cuda.get_device_properties(0).multi_processor_count


def tall(c, G, new, max_len=0):
    """max_q of a call on 128-row tiles, and its plan."""
    n = c.pages.shape[1] * c.page
    n = min(n, max_len) if max_len else n
    q = max_q_of_tall_tiles(len(c.lens), c.Hkv, G, max(max(new), 1), n, c.d, n_cu())
    return q, fwd_plan(len(c.lens), c.Hkv, G, q, n, c.d, n_cu())


def call(A, c, q, kind, new, max_q, out_dtype=torch.float32, **kw):
    """out and lse as float64; rows that no call writes hold 7."""
    gq = q.cuda() if torch.is_tensor(q) else R.torch_q(q, kind).cuda()
    out = torch.full(gq.shape, 7.0, dtype=out_dtype, device="cuda")
    lse = torch.full(gq.shape[:2], 7.0, device="cuda")
    A.cache_fwd(gq, dev_cache(A, c), dev(c.pages), dev(c.lens), cu=dev(cu_of(new)), max_q=max_q, out=out, lse=lse, **kw)
    return out.cpu().double().numpy(), lse.cpu().double().numpy()


def check(A, c, q, G, kind, new, max_q, out_dtype=torch.float32, max_len=0, **kw):
    o, l = call(A, c, q, kind, new, max_q, out_dtype, max_len=max_len, **kw)
    want, wl, bound, lb = R.attention(c, q, G, cu=cu_of(new), **kw)
    left = np.isnan(bound)
    assert np.all(o[left] == 7.0) and np.all(l[np.isnan(lb)] == 7.0)
    within(o[~left], want[~left], bound[~left] + (np.abs(want[~left]) * 2.0 ** -8 if out_dtype == torch.bfloat16 else 0.0))
    there = ~np.isnan(lb)
    assert np.array_equal(np.isinf(l[there]), np.isinf(wl[there]))
    there &= np.isfinite(wl)
    if there.any():
        within(l[there], wl[there], lb[there])
    return o, l


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("lens,new", [([40], [40]), ([300, 129, 5], [17, 129, 5]), ([500, 0, 260, 128], [1, 0, 33, 100]),
                                      ([1000, 90], [200, 3])])
def test_chunk(A, lens, new, d, page, kind, causal):
    G, Hkv = (3, 2) if d == 64 else (4, 2)
    rng = np.random.default_rng(sum(lens) + d + page)
    c = R.make_cache(rng, len(lens), Hkv, page, d, lens)
    q = R.make_queries(rng, sum(new) + 2, G * Hkv, d)      # two rows behind the last sequence
    max_q, plan = tall(c, G, new)
    log(f"tall chunk {lens} {new} d={d} page={page} {kind} causal={causal} max_q={max_q} ranges={plan.ranges}")
    check(A, c, q, G, kind, new, max_q, torch.bfloat16 if page == 64 else torch.float32, causal=causal)


# B, G, the bound on new tokens, keys, d, ranges on 256 compute units
SPLITS = [(2, 4, 400, 2000, 128, 4), (2, 8, 400, 4000, 64, 5), (1, 4, 200, 8000, 128, 16), (1, 8, 200, 16000, 64, 18)]


@pytest.mark.parametrize("page,kind", [(64, "bf16"), (128, "e4m3")])
@pytest.mark.parametrize("B,G,max_q,n,d,ranges", SPLITS)
def test_split_over_keys(A, B, G, max_q, n, d, ranges, page, kind):
    """Ranges and their merge (a row per workgroup beyond 8 of them), long sequences and short ones."""
    rng = np.random.default_rng(n + d)
    lens, new = [n, 140][:B], [40, 9][:B]
    c = R.make_cache(rng, B, 2, page, d, lens)
    plan = fwd_plan(B, 2, G, max_q, c.pages.shape[1] * page, d, n_cu())
    assert plan.rows == 128 and plan.ranges > 1 and (n_cu() != 256 or (plan.ranges > 8) == (ranges > 8))
    q = R.make_queries(rng, sum(new), 2 * G, d)
    log(f"tall split B={B} G={G} n={n} d={d} page={page} {kind} ranges={plan.ranges}")
    check(A, c, q, G, kind, new, max_q)
    # the last rows see fewer visits than the plan has ranges for
    c.lens[0] = n // 3
    check(A, c, q, G, kind, new, max_q, torch.bfloat16)


@pytest.mark.parametrize("n,d,ranges", [(16500, 64, 9), (16500, 128, 9), (3000, 64, 2)])
def test_split_of_single_tokens(A, n, d, ranges):
    """The merge of 16-row tiles with more than 8 ranges (a row per workgroup) and with fewer."""
    rng = np.random.default_rng(n + d)
    lens = [n, 140, 0, 1]
    c = R.make_cache(rng, 4, 1, 128, d, lens)
    plan = fwd_plan(4, 1, 5, 1, c.pages.shape[1] * 128, d, n_cu())
    assert plan.rows == 16 and plan.ranges > 1 and (n_cu() != 256 or (plan.ranges > 8) == (ranges > 8))
    q = R.make_queries(rng, 4, 5, d)
    log(f"split n={n} d={d} ranges={plan.ranges}")
    check(A, c, q, 5, "bf16", [1] * 4, 1)
    check(A, c, q, 5, "e4m3", [1] * 4, 1, torch.bfloat16)


@pytest.mark.parametrize("d,page", [(64, 64), (128, 64), (128, 128)])
def test_pages_that_are_none_and_lengths_outside_the_table(A, d, page):
    rng = np.random.default_rng(9 + d)
    c = R.make_cache(rng, 4, 2, page, d, [512, 130, 64, 300])
    c.pages[0, 2], c.pages[1, 130 // page], c.pages[2, 0] = -1, 1 << 30, c.n_pages
    new = [200, 2, 1, 150]
    q = R.make_queries(rng, sum(new), 4, d)
    max_q, _ = tall(c, 2, new)
    log(f"tall bad pages d={d} page={page}")
    _, lse = check(A, c, q, 2, "bf16", new, max_q)
    assert np.isinf(lse[202]).all()                        # its only page is none
    c.lens[0], c.lens[3] = 600, -5                         # past the table; no key, positions below 0
    check(A, c, q, 2, "e4m3", new, max_q)


def test_bound_on_the_length(A):
    """Keys from max_len on are not seen; positions stay."""
    rng = np.random.default_rng(10)
    c = R.make_cache(rng, 2, 2, 64, 64, [290, 64])
    new = [70, 64]
    q = R.make_queries(rng, sum(new), 4, 64)
    max_q, _ = tall(c, 2, new, 290)
    want, wl, bound, lb = R.attention(c, q, 2, cu=cu_of(new))
    check(A, c, q, 2, "bf16", new, max_q, max_len=290)
    max_q, _ = tall(c, 2, new, 250)
    o, l = call(A, c, q, "bf16", new, max_q, max_len=250)
    same = np.r_[:30, 70:134]                              # rows that see no key past 250
    within(o[same], want[same], bound[same])
    within(l[same], wl[same], lb[same])
    # the others see the 250 first keys, as a query that is not causal does among 250
    c.lens[0] = 250
    w2, l2, b2, lb2 = R.attention(c, q[30:70], 2, cu=np.array([0, 40, 40]), causal=False)
    within(o[30:70], w2, b2)
    within(l[30:70], l2, lb2)


def test_queries_with_strides(A):
    rng = np.random.default_rng(12)
    c = R.make_cache(rng, 2, 2, 128, 128, [300, 77])
    new = [50, 60]
    q = R.make_queries(rng, 110, 8, 128)
    max_q, _ = tall(c, 4, new)
    t = R.torch_q(q, "bf16").cuda()
    wide = torch.zeros((110, 16, 128), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:11] = t
    turned = t.transpose(0, 1).contiguous().transpose(0, 1)     # heads outermost
    want = call(A, c, t, "bf16", new, max_q)
    for x in (wide[:, 3:11], turned):
        got = call(A, c, x, "bf16", new, max_q)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 20), (128, 64, 1, 130), (64, 128, 8, 40)])
def test_nan_values_reach_the_rows_that_see_them(A, d, page, G, new, kind):
    """NaN codes of K and V in a chunk: rows before them are as without, rows from them on are NaN (V: in
    the NaN's channel alone)."""
    rng = np.random.default_rng(d + new)
    n = 150 + new
    c = R.make_cache(rng, 1, 1, page, d, [n])
    q = R.make_queries(rng, new, G, d)
    max_q, _ = tall(c, G, [new])
    want, wl, bound, lb = R.attention(c, q, G)
    t = n - new // 2                                   # a key that the first half of the rows does not see
    pid, slot = int(c.pages[0, t // page]), t % page
    log(f"tall nan d={d} page={page} G={G} new={new} {kind}")
    first = t - (n - new)                              # the first row that sees it
    c.v[pid, 0, slot, 5] = 0x7F
    c.v[pid, 0, slot, d - 1] = 0xFF
    o, l = call(A, c, q, kind, [new], max_q)
    hit = np.zeros(o.shape, dtype=bool)
    hit[first:, :, [5, d - 1]] = True
    assert np.array_equal(np.isnan(o), hit)
    within(np.where(hit, 0, o), np.where(hit, 0, want), bound)
    within(l, wl, lb)
    # a NaN in K: the rows that see it have a NaN score
    c.k[pid, 0, slot, 3] = 0x7F
    o, l = call(A, c, q, kind, [new], max_q)
    assert np.isnan(o[first:]).all() and np.isnan(l[first:]).all()
    within(o[:first], want[:first], bound[:first])
    within(l[:first], wl[:first], lb[:first])


def test_queries_that_are_not_finite_stay_in_their_rows(A):
    rng = np.random.default_rng(77)
    c = R.make_cache(rng, 2, 1, 64, 64, [300, 90])
    new = [40, 50]
    q = R.make_queries(rng, 90, 4, 64)
    max_q, _ = tall(c, 4, new)
    want, wl, bound, lb = R.attention(c, q, 4, cu=cu_of(new))
    t = R.torch_q(q, "bf16")
    t[0, 1, 7], t[35, 2, 3], t[60, 0, 0] = float("nan"), float("inf"), float("-inf")
    o, l = call(A, c, t, "bf16", new, max_q)
    bad = np.zeros((90, 4), dtype=bool)
    bad[0, 1] = bad[35, 2] = bad[60, 0] = True
    assert np.isnan(o[bad]).all() and np.isnan(l[bad]).all()
    within(o[~bad], want[~bad], bound[~bad])
    within(l[~bad], wl[~bad], lb[~bad])


def far_cache(rng, page, d, lens):
    """Blocks whose scores lie hundreds of powers of two apart and whose values do too: where a
    row's near blocks have a zero code, its far ones are what is left."""
    c = R.make_cache(rng, len(lens), 2, page, d, lens)
    c.ks[:] = rng.integers(118, 133, c.ks.shape)
    c.vs[:] = rng.choice([20, 60, 100, 127, 180, 200], c.vs.shape)
    return c


def check_far(A, c, q, G, kind, new, max_q):
    """As check, with FP32's range: sums below 2^-100 (each of n <= 2^11 keys drops what lies below
    2^-126 as an FP32 number, or is of a group below 2^(-119 - 119) with values of at most 2^83; by
    l >= 1/2) are not looked at."""
    o, l = call(A, c, q, kind, new, max_q, sm_scale=0.25, q_descale=0.75)
    want, wl, bound, lb = R.attention(c, q, G, cu=cu_of(new), sm_scale=0.25, q_descale=0.75)
    within(o, want, bound + 2.0 ** -100)
    within(l, wl, lb)
    return want, bound


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 128), (128, 64)])
def test_far_groups_of_large_values(A, d, page, kind):
    rng = np.random.default_rng(8)
    new = [60, 41]
    c = far_cache(rng, page, d, [700, 450])
    q = R.make_queries(rng, sum(new), 4, d)
    max_q, _ = tall(c, 2, new)
    log(f"tall far groups d={d} page={page} {kind}")
    check_far(A, c, q, 2, kind, new, max_q)


@pytest.mark.parametrize("B,G,max_q,n,d,rows", [(2, 4, 1, 2000, 64, 16), (2, 4, 1, 2000, 128, 16), (2, 4, 400, 2000, 128, 128),
                                                (2, 8, 12, 500, 64, 16)])
def test_far_groups_in_ranges_and_waves(A, B, G, max_q, n, d, rows):
    """The same where waves, and ranges with a merge, stand at their own powers of two."""
    rng = np.random.default_rng(n + d + max_q)
    new = [min(max_q, 30), 1]
    c = far_cache(rng, 64, d, [n, 130])
    plan = fwd_plan(B, 2, G, max_q, c.pages.shape[1] * 64, d, n_cu())
    assert plan.rows == rows and (plan.ranges > 1) == (n == 2000)
    q = R.make_queries(rng, sum(new), 2 * G, d)
    log(f"far groups G={G} max_q={max_q} n={n} d={d} ranges={plan.ranges}")
    check_far(A, c, q, G, "bf16", new, max_q)


@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 1), (128, 64, 4, 130), (64, 128, 8, 40)])
def test_factors_below_fp32_leave_masked_keys_out(A, d, page, G, new):
    """Blocks of zeros (scale 2^-127) and a small descale: scores of 0, and keys that a row does not see
    get nothing."""
    rng = np.random.default_rng(d + G)
    n = 200 + new
    c = R.make_cache(rng, 1, 1, page, d, [n])
    c.k[:], c.ks[:] = 0, 0
    q = R.make_queries(rng, new, G, d)
    max_q, _ = tall(c, G, [new])
    log(f"tall small factor d={d} page={page} G={G} new={new}")
    check(A, c, q, G, "bf16", [new], max_q, sm_scale=2.0 ** -10, q_descale=2.0 ** -30)


@pytest.mark.parametrize("d,page,G,new", [(64, 64, 2, 6), (128, 128, 4, 1), (128, 64, 4, 130), (64, 128, 8, 40)])
def test_scores_beyond_two_to_the_thirty(A, d, page, G, new):
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
    max_q, _ = tall(c, G, [new])
    log(f"tall far scores d={d} page={page} G={G} new={new}")
    o, l = call(A, c, q, "bf16", [new], max_q)
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
    within(o.reshape(-1, d), p @ v, np.broadcast_to(2.0 ** -10 * np.abs(v).max(), (new * G, d)))
    wl = (top[:, 0] + np.log2((x == top).sum(1))) * math.log(2.0)
    within(l.reshape(-1), wl, 2.0 ** -22 * np.abs(wl))


def test_captured_chunk_follows_the_lengths(A):
    """A split chunk on 128-row tiles captured once and replayed while lens and the tokens change, beside
    eager work, equals eager calls."""
    rng = np.random.default_rng(13)
    c = R.make_cache(rng, 2, 2, 128, 128, [2000, 700])
    args = dev_cache(A, c), dev(c.pages)
    max_q = 400
    assert fwd_plan(2, 2, 4, max_q, c.pages.shape[1] * 128, 128, n_cu()).rows == 128
    assert fwd_plan(2, 2, 4, max_q, c.pages.shape[1] * 128, 128, n_cu()).ranges > 1
    q = R.torch_q(R.make_queries(rng, 90, 8, 128), "bf16").cuda()
    lens, cu = dev(c.lens), dev(cu_of([40, 50]))
    steps = [([2000, 700], [40, 50]), ([900, 50], [60, 30]), ([1, 699], [1, 89]), ([1999, 0], [90, 0])]
    eager = []
    for n, new in steps:
        eager.append([x.clone() for x in A.cache_fwd(q, *args, dev(np.array(n, np.int32)), cu=dev(cu_of(new)), max_q=max_q)])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = A.cache_fwd(q, *args, lens, cu=cu, max_q=max_q)
    for i, (n, new) in enumerate(steps):
        log(f"replay {i}")
        lens.copy_(dev(np.array(n, np.int32)))
        cu.copy_(dev(cu_of(new)))
        out.fill_(3.0)
        graph.replay()
        A.cache_fwd(q, *args, lens, cu=cu, max_q=max_q)
        torch.cuda.synchronize()
        t = sum(new)
        assert torch.equal(out[:t], eager[i][0][:t]) and torch.equal(lse[:t], eager[i][1][:t])
        assert bool((out[t:] == 3.0).all())


@pytest.mark.parametrize("byte", [0, 200, 255])
@pytest.mark.parametrize("max_q", [1, 16, 0])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_pages_behind_the_length_are_not_looked_at(A, d, max_q, byte):
    """Pages reserved for later tokens, whose codes and scale bytes nobody has written: a visit of 128 keys
    holds two pages of 64.  max_q 0: tiles of 128 rows."""
    rng = np.random.default_rng(d + max_q)
    lens, new = [40, 190, 64], [1, min(max(max_q, 1), 7), 1]
    c = R.make_cache(rng, 3, 2, 64, d, [n + 64 for n in lens])
    c.lens[:] = lens
    if max_q == 0:
        new = [30, 50, 1]
        max_q, _ = tall(c, 2, new)
    for b, n in enumerate(lens):
        later = c.pages[b, -(-n // 64):]
        later = later[later >= 0]
        assert later.size
        c.k[later], c.v[later], c.ks[later], c.vs[later] = 0x7F, 0x7F, 127, 127
        c.k[c.pages[b, n // 64], :, n % 64:], c.v[c.pages[b, n // 64], :, n % 64:] = 0x7F, 0x7F
    q = R.make_queries(rng, sum(new), 4, d)
    log(f"scales behind the length d={d} max_q={max_q} byte={byte}")
    o, l = check(A, c, q, 2, "bf16", new, max_q)
    for b, n in enumerate(lens):
        later = c.pages[b, -(-n // 64):]
        c.ks[later[later >= 0]], c.vs[later[later >= 0]] = byte, byte
    o2, l2 = call(A, c, q, "bf16", new, max_q)
    assert np.array_equal(o, o2) and np.array_equal(l, l2)


@pytest.mark.parametrize("d,page,G", [(64, 64, 2), (128, 128, 4)])
@pytest.mark.parametrize("lens,new,wide", [([25, 9, 300], [40, 9, 30], False), ([25, 9, 300], [40, 9, 30], True), ([2], [3], False),
                                           ([130], [200], True), ([0, 5], [7, 7], False), ([700, 20], [12, 24], False)])
def test_tokens_before_position_0_see_nothing(A, lens, new, wide, d, page, G):
    """A padded batch: more new tokens than the sequence has, not causal.  The others see every key, and the
    weights count the others alone.  wide: tiles of 128 rows."""
    rng = np.random.default_rng(sum(lens) + d)
    c = R.make_cache(rng, len(lens), 2, page, d, lens)
    c.v[c.pages[0, 0], :, 1, 5] = 0x7F                   # a NaN that nobody else sees
    q = R.make_queries(rng, sum(new), 2 * G, d)
    max_q = tall(c, G, new)[0] if wide else max(new)
    cu = cu_of(new)
    log(f"before 0: {lens} {new} d={d} max_q={max_q}")
    want, wl, bound, lb = R.attention(c, q, G, cu=cu, causal=False)
    before = np.concatenate([np.arange(n - m, n) < 0 for n, m in zip(lens, new)])
    want[before], bound[before], wl[before], lb[before] = 0, 0, -np.inf, 0
    o, l = call(A, c, q, "bf16", new, max_q, causal=False)
    hit = np.isnan(want)
    assert np.array_equal(np.isnan(o), hit)
    within(np.where(hit, 0, o), np.where(hit, 0, want), np.where(hit, 0, bound))
    assert np.array_equal(np.isinf(l), np.isinf(wl))
    fin = np.isfinite(wl)
    if fin.any():
        within(l[fin], wl[fin], lb[fin])
    # weights of the visible rows; lse of the others as a caller of another library might give it
    n_w = c.pages.shape[1] * page
    lse = np.where(fin, wl, 0.0).astype(np.float32)
    w = torch.zeros((len(lens), 2, n_w), device="cuda")
    A.cache_weights(R.torch_q(q, "bf16").cuda(), dev(lse), dev_cache(A, c), dev(c.pages), dev(c.lens), w, cu=dev(cu), max_q=max_q, causal=False)
    ww = R.weights(c, q, np.where(fin, lse, -np.inf), G, n_w, cu=cu, causal=False)
    within(w.cpu().double().numpy(), ww, 2.0 ** -17 * ww)


@pytest.mark.parametrize("d,page,G,lens,new,max_q,first,rows", [
    (64, 64, 2, [60, 300], [20, 3], 8, 0, 16), (128, 128, 4, [200, 9, 70], [60, 9, 1], 5, 3, 16),
    (64, 128, 8, [1000, 40], [900, 40], 700, 5, 128), (128, 64, 8, [900, 3], [450, 1], 400, 0, 128)])
def test_tokens_beyond_max_q_are_left_out(A, d, page, G, lens, new, max_q, first, rows):
    """More new tokens than max_q says: the first max_q are done at their places, the rows of the others stay
    as they were, and so do rows before the first sequence's."""
    rng = np.random.default_rng(d + max_q)
    c = R.make_cache(rng, len(lens), 2, page, d, lens)
    n = c.pages.shape[1] * page
    assert fwd_plan(len(lens), 2, G, max_q, n, d, n_cu()).rows == rows
    q = R.make_queries(rng, first + sum(new) + 1, 2 * G, d)
    cu = (cu_of(new) + first).astype(np.int32)
    log(f"beyond max_q d={d} {lens} {new} max_q={max_q}")
    out = torch.full(q.shape, 7.0, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    gq, gc, pages, glens = R.torch_q(q, "bf16").cuda(), dev_cache(A, c), dev(c.pages), dev(c.lens)
    A.cache_fwd(gq, gc, pages, glens, cu=dev(cu), max_q=max_q, out=out, lse=lse)
    want, wl, bound, lb = R.attention(c, q, G, cu=cu, max_q=max_q)
    o, l = out.cpu().double().numpy(), lse.cpu().double().numpy()
    left = np.isnan(bound)
    assert left.any() and np.all(o[left] == 7.0) and np.all(l[np.isnan(lb)] == 7.0)
    within(o[~left], want[~left], bound[~left])
    within(l[~np.isnan(lb)], wl[~np.isnan(lb)], lb[~np.isnan(lb)])
    w = torch.zeros((len(lens), 2, n), device="cuda")
    A.cache_weights(gq, lse, gc, pages, glens, w, cu=dev(cu), max_q=max_q)
    ww = R.weights(c, q, l.astype(np.float32), G, n, cu=cu, max_q=max_q)
    within(w.cpu().double().numpy(), ww, 2.0 ** -17 * ww)
