"""Refusals of the cache calls at their edges, on the host (no GPU needed): nothing is launched."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest

from tests.cache_plan import fwd_plan
from tests.test_cache_abi import batch, cache, heads, rotation

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


GB = 1 << 36


def test_rope_of_too_many_threads_is_unsupported(A):
    """16 channels a thread; a launch holds less than 2^32 threads."""
    r = rotation(A)
    big = lambda T, H, d: A.attn_fp8_rope(heads(A), heads(A), T, H, d, r, None)  # noqa: E731
    for T, H, d in ((1 << 26, 64, 1024), (1 << 30, 32, 128), ((1 << 31) - 1, (1 << 31) - 16, 1024), (1 << 23, 128, 64)):
        assert big(T, H, d) == A.ATTN_ERR_UNSUPPORTED, (T, H, d)


@pytest.mark.parametrize("B,max_q,Hkv,Hq", [((1 << 31) - 1, 1 << 26, 1 << 16, 1 << 16), (1 << 12, 1 << 20, 8, 8), (1 << 18, 1, 32, 32),
                                            (1 << 16, 1 << 16, 1, 1 << 8)])
def test_append_of_too_many_threads_is_unsupported(A, B, max_q, Hkv, Hq):
    """A workgroup per block that can get tokens, KV head, and K or V, and those of q: products that pass
    64 bits in the first case."""
    b, x = batch(A, B=B, max_q=max_q, cu=MB, T=64), heads(A)
    q = x if Hq != Hkv else None
    assert A.attn_fp8_cache_append(cache(A, Hkv=Hkv), b, x, x, rotation(A), q, q, Hq, None) == A.ATTN_ERR_UNSUPPORTED


@pytest.mark.parametrize("B,max_q,Hkv,G", [((1 << 31) - 1, 1 << 24, 1 << 16, 1), (1 << 20, 1, 16, 4), (64, 1 << 22, 64, 4)])
def test_attention_of_too_many_threads_is_unsupported(A, B, max_q, Hkv, G):
    c, b, x = cache(A, Hkv=Hkv), batch(A, B=B, max_q=max_q, cu=MB, T=64), heads(A)
    assert A.attn_fp8_cache_fwd(c, b, x, Hkv * G, MB, 1, MB, 1, 0.1, 1.0, 0, None, 0, None) == A.ATTN_ERR_UNSUPPORTED
    assert A.attn_fp8_cache_workspace_bytes(c, b, Hkv * G, 0) == (A.ATTN_ERR_UNSUPPORTED, 0)


@pytest.mark.parametrize("B,Hkv", [((1 << 31) - 1, 1 << 16), (1 << 20, 16)])
def test_weights_of_too_many_threads_are_unsupported(A, B, Hkv):
    """A workgroup per (sequence, KV head) at least; the new tokens are not in its grid."""
    c, b, x = cache(A, Hkv=Hkv), batch(A, B=B, cu=MB, T=64, max_q=1 << 22), heads(A)
    assert A.attn_fp8_cache_weights(c, b, x, Hkv, MB, 1, 0.1, 1.0, 0, 4 * MB, 1 << 40, 1 << 20, None) == A.ATTN_ERR_UNSUPPORTED


def test_grids_of_a_plan(A):
    """The tiles' and the merge's launches: whole rounds of 8 workgroups, a row or a thread per 16 bytes."""
    class Grids(ctypes.Structure):
        _fields_ = [("tiles", ctypes.c_uint), ("merges", ctypes.c_uint), ("merge_rows", ctypes.c_int)]

    f = ctypes.CDLL(A.LIB_PATH)["_ZN4attn15cache_fwd_gridsEiiiiiRKNS_7FwdPlanERNS_8FwdGridsE"]
    f.restype = ctypes.c_int

    def grids(B, Hkv, G, max_q, n, d):
        p, g = fwd_plan(B, Hkv, G, max_q, n, d), Grids()
        return p, f(B, Hkv, G, max_q, d, ctypes.byref(p), ctypes.byref(g)), g

    for B, Hkv, G, max_q, n, d in ((1, 2, 4, 1, 777, 64), (3, 2, 5, 1, 16500, 128), (2, 2, 4, 400, 2000, 128), (1, 8, 4, 2048, 16384, 128)):
        p, st, g = grids(B, Hkv, G, max_q, n, d)
        wgs = B * Hkv * p.tiles * p.ranges
        rows = 1 if p.ranges > 8 else 1024 // d
        assert st == 0 and g.tiles == -(-wgs // 8) * 8 and g.merge_rows == rows
        assert g.merges == (0 if p.ranges == 1 else B * Hkv * -(-max_q * G // rows))
    # 2^24 tiles; 2^25 rows to merge one by one
    for a in ((1 << 18, 64, 1, 1, 128, 128), (64, 64, 4, 2048, 1 << 23, 128)):
        p, st, _ = grids(*a)
        assert st != 0, (a, p.rows, p.ranges)


def test_evict_of_too_many_threads_is_unsupported(A):
    def big(B, Hkv, budget):
        c, b = cache(A, Hkv=Hkv), batch(A, B=B, pages=GB, lens=2 * GB)
        return A.attn_fp8_cache_evict(c, b, c, 3 * GB, 4 * GB, 512, 512, budget, 4, 0, 1 << 61, 6 * GB, None, None)
    for a in ((1 << 21, 2, 64), (1 << 10, 1 << 10, 1 << 14), (1 << 25, 1 << 7, 64)):
        assert big(*a) == A.ATTN_ERR_UNSUPPORTED, a


@pytest.mark.parametrize("broken", [False, True])
def test_the_other_calls_do_not_need_the_native_module(A, tmp_path, broken):
    """Without _cache_binding.so (or with one that does not load) the package is there, and the cache calls
    say what to do."""
    package = tmp_path / "paper_2606_06521_amd"
    package.mkdir()
    here = os.path.dirname(A.__file__)
    for name in ("__init__.py", "attn_fp8.py"):
        shutil.copy(os.path.join(here, name), package / name)
    os.symlink(A.LIB_PATH, package / os.path.basename(A.LIB_PATH))
    if broken:
        (package / "_cache_binding.so").write_bytes(b"not a library")
    code = """
import torch
from paper_2606_06521_amd import attn_fp8 as A
assert A.__file__.startswith({0!r}), A.__file__
assert A.attn_fp8_version() > 0 and A.kv_cache(1, 1, 64, device="cpu").k.shape == (1, 1, 128, 64)
x = torch.zeros((1, 1, 64))
for call in (lambda: A.rope(x, x, x), lambda: A.cache_fwd(x, None, x, x), lambda: A.cache_append(None, x, x, x, x)):
    try:
        call()
    except ImportError as e:
        assert "__graft_entry__.build()" in str(e) and "_cache_binding" in str(e), e
    else:
        raise SystemExit("no error")
try:
    A.fwd(x, x, x)
except ValueError:
    print("fine")
""".format(str(tmp_path))
    r = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, capture_output=True, text=True, timeout=120,
                       env={**os.environ, "PYTHONPATH": str(tmp_path)})
    assert r.stdout == "fine\n", r.stderr
