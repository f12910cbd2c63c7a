"""Refusals of the cache calls at their edges, on the host (no GPU needed): nothing is launched."""
import pytest

from tests.test_cache_abi import batch, cache, heads

MB = 1 << 20   # addresses are never dereferenced


@pytest.fixture(scope="module")
def A():
    from paper_2606_06521_amd import attn_fp8
    return attn_fp8


def evict(A, **kw):
    """B = 2, W = 4, 2 heads, page 128: every array at an address of its own."""
    a = dict(pages=MB, lens=2 * MB, new_pages=3 * MB, w=4 * MB, sb=1024, sh=512, budget=64, kept=5 * MB, new_lens=6 * MB, nw=7 * MB)
    a.update(kw)
    b = batch(A, pages=a["pages"], lens=a["lens"])
    return A.attn_fp8_cache_evict(cache(A), b, cache(A), a["new_pages"], a["w"], a["sb"], a["sh"], a["budget"], 4, 0, a["kept"],
                                  a["new_lens"], a["nw"], None)


@pytest.mark.parametrize("kw", [
    dict(new_lens=2 * MB), dict(new_lens=2 * MB + 4), dict(new_lens=2 * MB - 4),                 # lens, one entry of two
    dict(new_lens=MB + 28), dict(new_lens=3 * MB + 4), dict(kept=4 * MB + 4 * (1024 + 512 + 511)), dict(kept=4 * MB - 4 * 255),
    dict(nw=4 * MB), dict(nw=5 * MB + 4 * 255), dict(new_lens=5 * MB + 4 * 255), dict(nw=6 * MB - 4 * 255),
    dict(kept=3 * MB), dict(kept=2 * MB + 4)])
def test_evict_refuses_outputs_over_inputs(A, kw):
    """Workgroups read lens while another has written new_lens, and so on."""
    assert evict(A, **kw) == A.ATTN_ERR_INVALID_ARG


def test_evict_takes_neighbours(A):
    """Arrays side by side are fine: here the call gets as far as its launch, which no GPU refuses."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch on made-up addresses")
    for kw in (dict(), dict(new_lens=2 * MB + 8), dict(new_lens=2 * MB - 8), dict(kept=4 * MB + 4 * (1024 + 512 + 512)),
               dict(kept=4 * MB - 4 * 256), dict(nw=5 * MB + 4 * 256), dict(nw=None)):
        assert evict(A, **kw) == A.ATTN_ERR_HIP, kw


def weights(A, sb, sh, B=2, Hkv=2):
    return A.attn_fp8_cache_weights(cache(A, Hkv=Hkv), batch(A, B=B, T=B), heads(A), 2 * Hkv, MB, 1, 0.1, 1.0, 0, 4 * MB, sb, sh, None)


@pytest.mark.parametrize("sb,sh,B,Hkv", [(0, 512, 2, 2), (512, 512, 2, 2), (1023, 512, 2, 2), (511, 1 << 20, 2, 2), (512, 1023, 2, 2),
                                         (512, 1024, 3, 2), (0, 512, 2, 1), (511, 512, 2, 1)])
def test_weights_refuses_rows_that_overlap(A, sb, sh, B, Hkv):
    """Two sequences that add to the same entries (512 of a row) would lose one another's sums."""
    assert weights(A, sb, sh, B, Hkv) == A.ATTN_ERR_INVALID_ARG


def test_weights_takes_either_order_of_rows(A):
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch on made-up addresses")
    for sb, sh, B, Hkv in ((1024, 512, 2, 2), (512, 1024, 2, 2), (512, 1536, 3, 2), (0, 512, 1, 2), (512, 512, 2, 1), (1 << 62, 1 << 40, 4, 2)):
        assert weights(A, sb, sh, B, Hkv) == A.ATTN_ERR_HIP, (sb, sh, B, Hkv)
