"""The 64-bit definitions of attention over parts of the cache against each other and against cache_ref
(CPU): lists of all blocks are the whole cache; the choice keeps the page that holds the largest score."""
import numpy as np

from tests import cache_ref as R
from tests import parts_ref as P


def test_lists_of_all_blocks_are_the_whole_cache():
    rng = np.random.default_rng(1)
    for d, page, run in ((64, 64, 3), (128, 128, 40)):
        c = R.make_cache(rng, 2, 2, page, d, [333, 140])
        q = R.make_queries(rng, 44, 4, d)
        cu = np.array([0, 40, 43], dtype=np.int32)
        W = c.pages.shape[1]
        blocks = np.broadcast_to(np.arange(W)[::-1], (2, -(-40 // run), 2, W))
        a, b = P.attention(c, q, blocks, 2, run=run, cu=cu, max_q=40), R.attention(c, q, 2, cu=cu)
        for x, y in zip(a[:2], b[:2]):
            assert np.array_equal(np.isnan(x), np.isnan(y))
            assert np.allclose(x, y, rtol=1e-12, atol=1e-12, equal_nan=True)


def test_bounds_hold_every_score():
    """No key of a page scores above the page's bound, for queries that eight bits hold."""
    rng = np.random.default_rng(2)
    c = R.make_cache(rng, 1, 1, 64, 64, [640])
    b = P.bounds(c, np.zeros((c.n_pages, 1, 2, 64)), max_q=640)
    q = rng.integers(-127, 128, (5, 64)).astype(np.float64)
    k, e, _ = c.keys(0, 0, "k")
    s = (q @ k.T).reshape(5, 10, 64)
    lo, hi = b[c.pages[0], 0, 0], b[c.pages[0], 0, 1]
    u = np.maximum(q[:, None] * lo, q[:, None] * hi).sum(2)
    assert (s.max(2) <= u).all()


def test_the_choice_on_a_page_of_its_own():
    rng = np.random.default_rng(3)
    c = R.make_cache(rng, 1, 2, 64, 64, [64 * 20])
    q = rng.standard_normal((1, 4, 64))
    far = int(c.pages[0, 13])
    c.k[far, 1, 17] = R.encode(np.sign(q[0, 2]) * 448.0)         # a key along head 2's query, of KV head 1
    b = P.bounds(c, np.zeros((c.n_pages, 2, 2, 64)), max_q=1280)
    got = P.select(c, q, b, 2, 1, n_first=0, n_last=0)
    assert got[0, 0, 1].tolist() == [13]
