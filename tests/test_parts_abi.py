"""C ABI and binding of attention over parts of the cache, on the host (no GPU needed): the header's
symbols are exported, and bad arguments are refused before any HIP call."""
import ctypes
import os
import re
import shutil
import subprocess
import sys

import pytest
import torch

from tests.cache_plan import Plan
from tests.test_cache_abi import FAKE, QUERIES, SIZES, TOKENS, batch, cache, changed, heads

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "attn_fp8_parts.h")


@pytest.fixture(scope="module")
def A():
    from paper_2606_06521_amd import attn_fp8
    return attn_fp8


def test_exports_every_declared_symbol(A):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"^int (attn_fp8_\w+)\(", text, flags=re.M)))
    assert names == ["attn_fp8_cache_blocks_workspace_bytes", "attn_fp8_cache_bounds", "attn_fp8_cache_fwd_blocks",
                     "attn_fp8_cache_fwd_shared", "attn_fp8_cache_select", "attn_fp8_cache_select_workspace_bytes",
                     "attn_fp8_cache_shared_workspace_bytes"]
    lib = ctypes.CDLL(A.LIB_PATH)
    for n in names:
        assert hasattr(lib, n) and hasattr(A, n), n


def test_header_is_plain_c(A, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text(r'''
#include <stdio.h>
#include "attn_fp8_parts.h"
int main(void) {
    size_t a = 7, b = 7;
    attn_fp8_cache c = {0, 0, 0, 0, 0, 1, 128, 128};
    attn_fp8_batch t = {0, 0, 0, 0, 4, 0, 1};
    int x = attn_fp8_cache_blocks_workspace_bytes(&c, &t, 2, 3, 1, &a);
    int y = attn_fp8_cache_shared_workspace_bytes(&c, &t, 2, 2, 0, &b);
    printf("%d %d %zu %zu\n", x, y, a, b);
    return 0;
}
''')
    exe, libdir = tmp_path / "use", os.path.dirname(A.LIB_PATH)
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-pedantic-errors", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe), "-L", libdir, "-lattn_fp8", "-Wl,-rpath," + libdir], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.stdout.split() == ["0", "0", "0", "0"]


@pytest.mark.parametrize("kind,kw,status", SIZES + TOKENS + [("a", dict(bounds=None), -1), ("a", dict(bounds=FAKE + 8), -1)])
def test_bounds_refuses(A, kind, kw, status):
    c, b, _, _ = changed(A, kind, kw)
    assert A.attn_fp8_cache_bounds(c, b, kw.get("bounds", FAKE) if kind == "a" else FAKE, None) == status


ATTENTION = [("a", dict(Hq=3), -1), ("a", dict(Hq=0), -1), ("a", dict(Hq=2 * 257), -2), ("a", dict(causal=2), -1)]
OUTPUTS = [("a", dict(out=None), -1), ("a", dict(out=FAKE + 8), -1), ("a", dict(out_type=2), -1), ("a", dict(lse=FAKE + 1), -1),
           ("a", dict(sm=0.0), -1), ("a", dict(sm=float("nan")), -1), ("a", dict(qd=float("inf")), -1), ("a", dict(ws=FAKE + 16), -1)]
LISTS = [("a", dict(blocks=None), -1), ("a", dict(blocks=FAKE + 2), -1), ("a", dict(take=0), -1), ("a", dict(run=0), -1),
         ("a", dict(run=-4), -1)]


@pytest.mark.parametrize("kind,kw,status", SIZES + TOKENS + QUERIES + ATTENTION + LISTS + [
    ("a", dict(bounds=None), -1), ("a", dict(bounds=FAKE + 4), -1), ("a", dict(n_first=-1), -1), ("a", dict(n_last=-1), -1),
    ("a", dict(n_first=2, n_last=2), -1), ("a", dict(n_first=(1 << 31) - 1, n_last=(1 << 31) - 1), -1), ("a", dict(take=16385), -2),
    ("a", dict(max_len=-1), -1), ("b", dict(W=16385), -2), ("a", dict(ws=FAKE + 16), -1), ("b", dict(W=5000), -1)])
def test_select_refuses(A, kind, kw, status):
    c, b, q, _ = changed(A, kind, kw)
    a = dict(Hq=4, bounds=FAKE, blocks=FAKE, take=3, run=1, n_first=1, n_last=1, causal=1, max_len=0, ws=None)
    a.update(kw if kind == "a" else {})
    assert A.attn_fp8_cache_select(c, b, q, a["Hq"], a["bounds"], a["blocks"], a["take"], a["run"], a["n_first"], a["n_last"], a["causal"],
                                   a["max_len"], a["ws"], 0, None) == status


@pytest.mark.parametrize("kind,kw,status", SIZES + TOKENS + QUERIES + ATTENTION + OUTPUTS + LISTS + [("a", dict(take=(1 << 19) + 1), -2)])
def test_blocks_refuses(A, kind, kw, status):
    c, b, q, _ = changed(A, kind, kw)
    a = dict(Hq=4, blocks=FAKE, take=3, run=1, out=FAKE, out_type=1, lse=FAKE, causal=1, sm=0.1, qd=1.0, ws=None)
    a.update(kw if kind == "a" else {})
    assert A.attn_fp8_cache_fwd_blocks(c, b, q, a["Hq"], a["blocks"], a["take"], a["run"], a["out"], a["out_type"], a["lse"], a["causal"],
                                       a["sm"], a["qd"], a["ws"], 0, None) == status


@pytest.mark.parametrize("kind,kw,status", SIZES + TOKENS + QUERIES + ATTENTION + OUTPUTS + [
    ("a", dict(shared=-1), -1), ("a", dict(shared=5), -1), ("a", dict(max_len=-1), -1)])
def test_shared_refuses(A, kind, kw, status):
    c, b, q, _ = changed(A, kind, kw)
    a = dict(Hq=4, shared=2, out=FAKE, out_type=1, lse=FAKE, causal=1, sm=0.1, qd=1.0, max_len=0, ws=None)
    a.update(kw if kind == "a" else {})
    assert A.attn_fp8_cache_fwd_shared(c, b, a["shared"], q, a["Hq"], a["out"], a["out_type"], a["lse"], a["causal"], a["sm"], a["qd"],
                                       a["max_len"], a["ws"], 0, None) == status


def test_workspace_queries_refuse(A):
    c, b = cache(A), batch(A)
    assert A._lib.attn_fp8_cache_blocks_workspace_bytes(c, b, 4, 3, 1, None) == -1
    assert A._lib.attn_fp8_cache_shared_workspace_bytes(c, b, 2, 4, 0, None) == -1
    assert A.attn_fp8_cache_blocks_workspace_bytes(c, b, 4, 0, 1) == (-1, 0)
    assert A._lib.attn_fp8_cache_select_workspace_bytes(c, b, 4, 3, 1, 0, None) == -1
    assert A.attn_fp8_cache_select_workspace_bytes(c, b, 4, 0, 1, 0) == (-1, 0)
    assert A.attn_fp8_cache_select_workspace_bytes(c, batch(A, W=16385), 4, 3, 1, 0) == (-2, 0)
    assert A.attn_fp8_cache_select_workspace_bytes(c, b, 4, 3, 1, 0) == (0, 0)
    assert A.attn_fp8_cache_blocks_workspace_bytes(c, b, 5, 3, 1) == (-1, 0)
    assert A.attn_fp8_cache_shared_workspace_bytes(c, b, 5, 4, 0) == (-1, 0)
    assert A.attn_fp8_cache_shared_workspace_bytes(c, b, -1, 4, 0) == (-1, 0)


def test_empty_batches_are_fine(A):
    for kw in (dict(B=0, T=0), dict(T=0)):
        c, b, q = cache(A), batch(A, **kw), heads(A)
        assert A.attn_fp8_cache_fwd_blocks(c, b, q, 4, FAKE, 3, 1, FAKE, 1, FAKE, 1, 0.1, 1.0, None, 0, None) == 0
        assert A.attn_fp8_cache_fwd_shared(c, b, 2, q, 4, FAKE, 1, FAKE, 1, 0.1, 1.0, 0, None, 0, None) == 0
        assert A.attn_fp8_cache_bounds(c, b, FAKE, None) == 0
        assert A.attn_fp8_cache_blocks_workspace_bytes(c, b, 4, 3, 1) == (0, 0)
        assert A.attn_fp8_cache_shared_workspace_bytes(c, b, 2, 4, 0) == (0, 0)
    # (a batch of sequences without new tokens still gets its lists, of -1)
    assert A.attn_fp8_cache_select(c, batch(A, B=0, T=0), q, 4, FAKE, FAKE, 3, 1, 1, 1, 1, 0, None, 0, None) == 0


@pytest.mark.parametrize("B,max_q,Hkv,G,run", [((1 << 31) - 1, 1, 1 << 16, 1, 1), (1 << 12, 1 << 20, 8, 1, 1), (1 << 18, 64, 8, 4, 8)])
def test_lists_of_too_many_threads_are_unsupported(A, B, max_q, Hkv, G, run):
    c, b, q = cache(A, Hkv=Hkv), batch(A, B=B, T=1 << 30, cu=FAKE, max_q=max_q), heads(A)
    assert A.attn_fp8_cache_select(c, b, q, Hkv * G, FAKE, FAKE, 3, run, 1, 1, 1, 0, None, 0, None) == -2
    assert A.attn_fp8_cache_fwd_blocks(c, b, q, Hkv * G, FAKE, 3, run, FAKE, 1, FAKE, 1, 0.1, 1.0, None, 0, None) == -2
    assert A.attn_fp8_cache_blocks_workspace_bytes(c, b, Hkv * G, 3, run) == (-2, 0)


def test_shared_of_too_many_rows_is_unsupported(A):
    c, q = cache(A), heads(A)
    b = batch(A, cu=FAKE, T=(1 << 23) + 1)
    assert A.attn_fp8_cache_fwd_shared(c, b, 2, q, 4, FAKE, 1, FAKE, 1, 0.1, 1.0, 0, FAKE, 1 << 40, None) == -2
    assert A.attn_fp8_cache_shared_workspace_bytes(c, b, 2, 4, 0) == (-2, 0)


class _Grids(ctypes.Structure):
    _fields_ = [("pre", ctypes.c_uint), ("own", ctypes.c_uint), ("merges", ctypes.c_uint), ("merge_rows", ctypes.c_int)]


def test_shared_ranges_fit_the_merge(A):
    """The merge keeps a reference for each range of a row in LDS; more are refused before a launch."""
    from tests.parts_ref import SharedPlan
    f = ctypes.CDLL(A.LIB_PATH)["_ZN4attn12shared_gridsEiiiiiRKNS_10SharedPlanERNS_11SharedGridsE"]
    f.restype = ctypes.c_int
    for a, b, fits in ((4096, 1024, True), (4096, 1025, False), (1, 1, True)):
        p = SharedPlan(Plan(16, 1, 128, a, 0), Plan(16, 1, 128, b, 0))
        g = _Grids()
        assert (f(1, 1, 1, 1, 128, ctypes.byref(p), ctypes.byref(g)) == 0) == fits


def test_binding_refuses_tensors_on_the_host(A):
    q, pages, lens = torch.zeros((1, 2, 64), dtype=torch.bfloat16), torch.zeros((1, 1), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    c = A.kv_cache(1, 1, 64, page=64, device="cpu")
    lists = torch.zeros((1, 1, 1, 1), dtype=torch.int32)
    bounds = A.key_bounds(1, 1, 64, device="cpu")
    for f in (lambda: A.cache_fwd_blocks(q, c, pages, lens, lists), lambda: A.cache_fwd_shared(q, c, pages, lens, 1),
              lambda: A.cache_select(q, c, pages, lens, bounds, 1, n_last=0), lambda: A.cache_bounds(c, pages, lens, bounds)):
        with pytest.raises(ValueError, match="on the GPU"):
            f()


def test_workspace_of_a_choice_holds_its_keys(A):
    """A split choice (few lists of many pages) keeps four bytes for each page of each list."""
    split = 0
    for B, W, max_q, run in ((1, 2047, 1, 1), (1, 16384, 40, 8), (2, 600, 1, 1), (64, 4000, 1, 1), (4, 300, 1, 1), (65, 4000, 1, 1), (4, 256, 1, 1)):
        st, n = A.attn_fp8_cache_select_workspace_bytes(cache(A, page=64), batch(A, B=B, W=W, T=B, max_q=max_q, cu=FAKE), 4, 3, run, 0)
        assert st == 0 and n in (0, B * 2 * -(-max_q // run) * W * 4)
        split += n > 0
    assert split == 5           # (not: more than 128 lists; pages that one workgroup's waves hold)


def test_workspace_of_a_choice_for_an_empty_batch():
    """No sequences, tables on both sides of the split's thresholds: no workspace and no division by the
    number of lists, and the call itself is a no-op.  In a process of its own, which such a division would end."""
    code = """
from paper_2606_06521_amd import attn_fp8 as A
from tests.test_cache_abi import FAKE, batch, cache, heads
for W in (0, 4, 256, 257, 512, 513, 600, 16384):
    for page in (64, 128):
        c = cache(A, page=page)
        for b in (batch(A, B=0, T=0, W=W), batch(A, B=0, T=0, W=W, cu=FAKE, max_q=40)):
            assert A.attn_fp8_cache_select_workspace_bytes(c, b, 4, 3, 8, 0) == (0, 0), (W, page)
            assert A.attn_fp8_cache_select(c, b, heads(A), 4, FAKE, FAKE, 3, 8, 1, 1, 1, 0, None, 0, None) == 0
        # (sequences without new tokens have lists, so their choice keeps its keys)
        st, n = A.attn_fp8_cache_select_workspace_bytes(c, batch(A, T=0, W=W), 4, 3, 1, 0)
        assert st == 0 and n == (2 * 2 * W * 4 if W > 256 else 0), (W, page, st, n)
print("done")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["done"], (r.returncode, r.stdout, r.stderr[-2000:])


@pytest.mark.parametrize("B,Hkv", [(1 << 23, 2), (1 << 8, 1 << 16), ((1 << 30) - 1, 1)])
def test_bounds_of_too_many_heads_are_unsupported(A, B, Hkv):
    for cu in (None, FAKE):
        assert A.attn_fp8_cache_bounds(cache(A, Hkv=Hkv), batch(A, B=B, T=B, cu=cu), FAKE, None) == -2
