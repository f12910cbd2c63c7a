"""The plan of the cache's attention on 256 compute units (host code; no GPU needed): which kernel
and split a call takes, and that the GPU tests of the splits name the ones there are."""
import pytest

from tests.cache_plan import fwd_plan, max_q_of_tall_tiles
from tests.test_gpu_cache_tiles import SPLITS


def test_the_gpu_tests_of_the_splits_reach_both_merges():
    few, many = set(), set()
    for B, G, max_q, n, d, ranges in SPLITS:
        for page in (64, 128):
            p = fwd_plan(B, 2, G, max_q, -(-n // page) * page, d)
            assert (p.rows, p.ranges) == (128, ranges)
        (many if ranges > 8 else few).add(d)
    assert few == many == {64, 128}
    for n, d, more in ((16500, 64, True), (16500, 128, True), (3000, 64, False)):
        p = fwd_plan(4, 1, 5, 1, -(-n // 128) * 128, d)
        assert p.rows == 16 and p.ranges > 1 and (p.ranges > 8) == more


@pytest.mark.parametrize("B,Hkv,G,max_q,n,d,rows", [
    (16, 8, 4, 1, 8192, 128, 16), (1, 8, 4, 1, 131001, 128, 16), (4, 2, 4, 1, 777, 64, 16),   # single tokens
    (1, 8, 4, 2048, 16384, 128, 128), (16, 8, 4, 24, 8192, 128, 128), (1, 8, 1, 256, 32768, 128, 128),   # chunks
    (16, 8, 4, 8, 8192, 128, 16), (1, 8, 1, 64, 32768, 128, 16),
])
def test_tiles_by_the_rows_of_a_call(B, Hkv, G, max_q, n, d, rows):
    assert fwd_plan(B, Hkv, G, max_q, n, d).rows == rows


def test_a_loose_bound_on_the_new_tokens_makes_tall_tiles():
    for B, Hkv, G, new, n, d in ((1, 1, 1, 1, 128, 64), (3, 2, 4, 40, 320, 128), (8, 8, 8, 5, 1000, 64)):
        q = max_q_of_tall_tiles(B, Hkv, G, new, n, d)
        assert q >= new and fwd_plan(B, Hkv, G, q, n, d).rows == 128


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [16, 128])
def test_workspace_holds_every_range_of_every_tile(d, rows):
    seen = 0
    for B in (1, 3, 64):
        for q in (1, 40, 700):
            for n in (100, 5000, 70000, 1 << 20):
                p = fwd_plan(B, 2, 4, q, n, d)
                if p.rows != rows:
                    continue
                seen += 1
                visits = -(-n // 128)
                assert p.tiles * p.rows >= q * 4 and p.chunk * p.ranges >= visits
                assert p.chunk <= (128 if rows == 16 else 512) and p.ranges <= 4096
                assert p.bytes == (0 if p.ranges == 1 else B * 2 * p.tiles * p.ranges * rows * (d + 2) * 4)
    assert seen >= 4
