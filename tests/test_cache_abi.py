"""The KV cache's C ABI and binding on the host (no GPU needed): the header's symbols are
exported, structures and enums match, and bad arguments are refused before any HIP call."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "attn_fp8_cache.h")
FAKE = 1 << 20   # never dereferenced: every case below fails validation first


@pytest.fixture(scope="module")
def A():
    from paper_2606_06521_amd import attn_fp8
    return attn_fp8


def test_exports_every_declared_symbol(A):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"^int (attn_fp8_\w+)\(", text, flags=re.M)))
    assert names == ["attn_fp8_cache_append", "attn_fp8_cache_evict", "attn_fp8_cache_fwd", "attn_fp8_cache_weights",
                     "attn_fp8_cache_workspace_bytes", "attn_fp8_rope"]
    lib = ctypes.CDLL(A.LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n
        assert hasattr(A, n), n
    for name in re.findall(r"\b(ATTN_(?:TYPE|ROPE)_\w+) =", text):
        assert int(re.search(name + r" = (\d+)", text).group(1)) == getattr(A, name), name


def test_header_is_plain_c_and_structures_match(A, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text(r'''
#include <stdio.h>
#include "attn_fp8_cache.h"
int main(void) {
    size_t n = 7;
    attn_fp8_cache c = {0, 0, 0, 0, 0, 1, 128, 128};
    attn_fp8_batch b = {0, 0, 0, 0, 4, 0, 1};
    int st = attn_fp8_cache_workspace_bytes(&c, &b, 2, 0, &n);
    printf("%zu %zu %zu %zu %d %zu\n", sizeof(attn_fp8_cache), sizeof(attn_fp8_batch), sizeof(attn_fp8_heads),
           sizeof(attn_fp8_rotation), st, n);
    return 0;
}
''')
    exe, libdir = tmp_path / "use", os.path.dirname(A.LIB_PATH)
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-pedantic-errors", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe), "-L", libdir, "-lattn_fp8", "-Wl,-rpath," + libdir], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    sizes = [ctypes.sizeof(t) for t in (A.attn_fp8_cache, A.attn_fp8_batch, A.attn_fp8_heads, A.attn_fp8_rotation)]
    assert r.stdout.split() == [str(x) for x in sizes + [0, 0]]


def cache(A, **kw):
    a = dict(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, n_pages=8, Hkv=2, page=128, d=128)
    a.update(kw)
    return A.attn_fp8_cache(*a.values())


def batch(A, **kw):
    a = dict(pages=FAKE, lens=FAKE, cu=None, B=2, W=4, T=2, max_q=1)
    a.update(kw)
    return A.attn_fp8_batch(*a.values())


def heads(A, **kw):
    a = dict(data=FAKE, st=1024, sh=128, type=A.ATTN_TYPE_BF16)
    a.update(kw)
    return A.attn_fp8_heads(*a.values())


def rotation(A, **kw):
    a = dict(table=FAKE, positions=FAKE, n_pos=64, rot=64, layout=0)
    a.update(kw)
    return A.attn_fp8_rotation(*a.values())


# what every call of a cache and a batch refuses (kind, change, status)
SIZES = [("c", dict(d=96), -2), ("c", dict(page=32), -2), ("c", dict(page=0), -1), ("c", dict(d=0), -1), ("c", dict(Hkv=0), -1),
         ("c", dict(n_pages=-1), -1), ("b", dict(B=-1), -1), ("b", dict(W=-1), -1), ("b", dict(T=-1), -1), ("b", dict(max_q=0), -1),
         ("b", dict(W=1 << 24), -2), ("b", dict(W=(1 << 19) + 1), -2), ("c", dict(k=None), -1), ("c", dict(v=None), -1), ("c", dict(ks=None), -1),
         ("c", dict(vs=None), -1), ("c", dict(k=FAKE + 8), -1), ("c", dict(v=FAKE + 1), -1), ("b", dict(pages=None), -1),
         ("b", dict(lens=None), -1), ("b", dict(lens=FAKE + 2), -1), ("b", dict(pages=FAKE + 1), -1)]
# and of the new tokens
TOKENS = [("b", dict(T=3), -1), ("b", dict(T=8), -1), ("b", dict(cu=FAKE + 2), -1)]
QUERIES = [("q", dict(data=None), -1), ("q", dict(data=FAKE + 8), -1), ("q", dict(st=1028), -1), ("q", dict(sh=4), -1),
           ("q", dict(st=-1024), -1), ("q", dict(type=0), -1), ("q", dict(type=2), -1), ("q", dict(type=9), -1)]


def changed(A, kind, kw):
    return (cache(A, **(kw if kind == "c" else {})), batch(A, **(kw if kind == "b" else {})),
            heads(A, **(kw if kind == "q" else {})), rotation(A, **(kw if kind == "r" else {})))


@pytest.mark.parametrize("kind,kw,status", SIZES + TOKENS + QUERIES + [
    ("a", dict(Hq=3), -1), ("a", dict(Hq=0), -1), ("a", dict(out=None), -1), ("a", dict(out=FAKE + 8), -1), ("a", dict(out_type=2), -1),
    ("a", dict(lse=FAKE + 1), -1), ("a", dict(causal=2), -1), ("a", dict(sm=0.0), -1), ("a", dict(sm=float("nan")), -1),
    ("a", dict(qd=float("inf")), -1), ("a", dict(qd=-1.0), -1), ("a", dict(max_len=-1), -1), ("a", dict(ws=FAKE + 16), -1)])
def test_fwd_refuses(A, kind, kw, status):
    c, b, q, _ = changed(A, kind, kw)
    a = dict(Hq=4, out=FAKE, out_type=1, lse=FAKE, causal=1, sm=0.1, qd=1.0, max_len=0, ws=None)
    a.update(kw if kind == "a" else {})
    assert A.attn_fp8_cache_fwd(c, b, q, a["Hq"], a["out"], a["out_type"], a["lse"], a["causal"], a["sm"], a["qd"],
                                a["max_len"], a["ws"], 0, None) == status


@pytest.mark.parametrize("kind,kw,status", SIZES + TOKENS + QUERIES + [
    ("a", dict(Hq=5), -1), ("a", dict(lse=None), -1), ("a", dict(w=None), -1), ("a", dict(w=FAKE + 2), -1), ("a", dict(sh=511), -1),
    ("a", dict(sb=-1), -1), ("a", dict(sm=-0.1), -1), ("a", dict(causal=-1), -1)])
def test_weights_refuses(A, kind, kw, status):
    c, b, q, _ = changed(A, kind, kw)
    a = dict(Hq=4, lse=FAKE, causal=1, sm=0.1, w=FAKE, sb=1024, sh=512)
    a.update(kw if kind == "a" else {})
    assert A.attn_fp8_cache_weights(c, b, q, a["Hq"], a["lse"], a["causal"], a["sm"], 1.0, 0, a["w"], a["sb"], a["sh"], None) == status


@pytest.mark.parametrize("kind,kw,status", SIZES + TOKENS + [
    ("q", dict(data=None), -1), ("q", dict(type=3), -1), ("q", dict(type=0), -1), ("q", dict(sh=1), -1),
    ("r", dict(table=None), -1), ("r", dict(table=FAKE + 4), -1), ("r", dict(rot=24), -2), ("r", dict(rot=0), -1),
    ("r", dict(rot=144), -1), ("r", dict(layout=2), -1), ("r", dict(n_pos=0), -1), ("r", dict(positions=FAKE + 1), -1),
    ("a", dict(k=False), -1), ("a", dict(v=False), -1), ("a", dict(r=False, q=True), -1), ("a", dict(q=True, Hq=0), -1),
    ("a", dict(q=True, lone=True), -1), ("a", dict(q=True, qtype=0), -1)])
def test_append_refuses(A, kind, kw, status):
    c, b, k, r = changed(A, kind, kw)
    a = dict(k=True, v=True, r=True, q=False, Hq=4, lone=False, qtype=1)
    a.update(kw if kind == "a" else {})
    v = heads(A)
    q = heads(A, type=a["qtype"]) if a["q"] else None
    o = None if a["lone"] else q
    assert A.attn_fp8_cache_append(c, b, k if a["k"] else None, v if a["v"] else None, r if a["r"] else None, q, o, a["Hq"],
                                   None) == status


@pytest.mark.parametrize("kind,kw,status", SIZES + [
    ("t", dict(Hkv=4), -1), ("t", dict(page=64), -1), ("t", dict(d=64), -1), ("t", dict(k=None), -1), ("t", dict(v=FAKE + 4), -1),
    ("a", dict(np=None), -1), ("a", dict(w=None), -1), ("a", dict(sh=511), -1), ("a", dict(budget=0), -1),
    ("a", dict(budget=(1 << 20) + 1), -2), ("a", dict(sink=-1), -1), ("a", dict(recent=-1), -1), ("a", dict(kept=None), -1),
    ("a", dict(lens=None), -1), ("a", dict(nw=FAKE + 2), -1), ("a", dict(kept=FAKE + 1), -1)])
def test_evict_refuses(A, kind, kw, status):
    c, b, _, _ = changed(A, kind, kw)
    t = cache(A, **(kw if kind == "t" else {}))
    a = dict(np=FAKE, w=FAKE, sb=1024, sh=512, budget=64, sink=4, recent=0, kept=FAKE, lens=FAKE, nw=None)
    a.update(kw if kind == "a" else {})
    assert A.attn_fp8_cache_evict(c, b, t, a["np"], a["w"], a["sb"], a["sh"], a["budget"], a["sink"], a["recent"], a["kept"],
                                  a["lens"], a["nw"], None) == status


@pytest.mark.parametrize("kind,kw,status", [
    ("x", dict(data=None), -1), ("x", dict(data=FAKE + 4), -1), ("x", dict(type=3), -1), ("x", dict(st=1), -1), ("o", dict(type=0), -1),
    ("o", dict(data=None), -1), ("r", dict(rot=8), -2), ("r", dict(rot=144), -1), ("r", dict(positions=None), -1),
    ("r", dict(layout=-1), -1), ("a", dict(T=-1), -1), ("a", dict(H=-1), -1), ("a", dict(d=0), -1), ("a", dict(d=72), -2),
    ("a", dict(d=2048), -2)])
def test_rope_refuses(A, kind, kw, status):
    a = dict(T=2, H=2, d=128)
    a.update(kw if kind == "a" else {})
    x, o = heads(A, **(kw if kind == "x" else {})), heads(A, **(kw if kind == "o" else {}))
    assert A.attn_fp8_rope(x, o, a["T"], a["H"], a["d"], rotation(A, **(kw if kind == "r" else {})), None) == status


def test_empty_calls_are_no_ops(A):
    none = dict(k=None, v=None, ks=None, vs=None)
    for kw in (dict(B=0, T=0), dict(T=0)):
        b, c, q, r = batch(A, pages=None, lens=None, **kw), cache(A, **none), heads(A, data=None), rotation(A, table=None)
        assert A.attn_fp8_cache_fwd(c, b, q, 4, None, 1, None, 1, 0.1, 1.0, 0, None, 0, None) == 0
        assert A.attn_fp8_cache_append(c, b, q, q, r, None, None, 0, None) == 0
        assert A.attn_fp8_cache_weights(c, b, q, 4, None, 1, 0.1, 1.0, 0, None, 0, 0, None) == 0
        assert A.attn_fp8_cache_workspace_bytes(c, b, 4, 0) == (0, 0)
    assert A.attn_fp8_cache_evict(cache(A, **none), batch(A, B=0), cache(A, **none), None, None, 0, 0, 1, 0, 0, None, None, None, None) == 0
    assert A.attn_fp8_rope(heads(A, data=None), heads(A, data=None), 0, 2, 128, rotation(A), None) == 0
    assert A._lib.attn_fp8_cache_workspace_bytes(cache(A), batch(A), 4, 0, None) == -1
    assert A.attn_fp8_cache_workspace_bytes(cache(A), batch(A), 5, 0)[0] == -1


def test_binding_refuses_host_tensors(A):
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    i = torch.zeros((2,), dtype=torch.int32)
    c = A.kv_cache(1, 2, 64, page=64, device="cpu")
    p = torch.zeros((2, 1), dtype=torch.int32)
    t = A.rope_table(4, 64, device="cpu")
    w = torch.zeros((2, 2, 64))
    for call in (lambda: A.rope(x, t, i), lambda: A.cache_append(c, x, x, p, i), lambda: A.cache_fwd(x, c, p, i),
                 lambda: A.cache_weights(x, torch.zeros((2, 2)), c, p, i, w), lambda: A.cache_evict(c, p, i, w, c, p, 8)):
        with pytest.raises(ValueError):
            call()


def test_rope_table_is_the_formula_and_refuses(A):
    def angles(t):
        return np.arctan2(t[..., 1].double().numpy(), t[..., 0].double().numpy())
    p = np.arange(50)[:, None]
    i = np.arange(16)
    f = 10000.0 ** (-2 * i / 32)
    wrap = lambda a: (a + np.pi) % (2 * np.pi) - np.pi  # noqa: E731
    near = lambda a, b: np.abs(wrap(a - b)).max() < 1e-6  # noqa: E731  (two FP32 roundings of unit size)
    assert near(angles(A.rope_table(50, 32, device="cpu")), p * f)
    assert near(angles(A.rope_table(50, 32, scaling="linear", factor=4.0, device="cpu")), p * f / 4)
    g = (10000.0 * 4.0 ** (32 / 30)) ** (-2 * i / 32)
    assert near(angles(A.rope_table(50, 32, scaling="base", factor=4.0, device="cpu")), p * g)
    assert abs(g[-1] / f[-1] - 0.25) < 1e-12 and g[0] == f[0]
    turns = 2048 * f / (2 * np.pi)
    keep = np.clip((turns - 1) / 31, 0, 1)
    assert near(angles(A.rope_table(50, 32, scaling="ramp", factor=4.0, original=2048, device="cpu")), p * (f * keep + f / 4 * (1 - keep)))
    # far positions: angles in 64 bits
    far = A.rope_table(1 << 17, 16, device="cpu")[-1]
    assert near(angles(far), ((1 << 17) - 1) * 10000.0 ** (-2 * np.arange(8) / 16))
    for kw in (dict(rot=3), dict(rot=0), dict(n_pos=0), dict(factor=0.0), dict(scaling="other"), dict(scaling="ramp"),
               dict(scaling="base", rot=2), dict(base=-1.0)):
        a = dict(n_pos=4, rot=32, device="cpu")
        a.update(kw)
        with pytest.raises(ValueError):
            A.rope_table(a.pop("n_pos"), a.pop("rot"), **a)


def test_sizes_past_32_bit_positions_and_caches_without_pages_are_refused(A):
    """Past 2^30 tokens a key's distance from a position would wrap; an eviction loads page 0
    for rows that have none."""
    b, q, r = batch(A, cu=FAKE, T=(1 << 30) + 1), heads(A), rotation(A)
    assert A.attn_fp8_cache_fwd(cache(A), b, q, 4, FAKE, 1, FAKE, 1, 0.1, 1.0, 0, None, 0, None) == -2
    assert A.attn_fp8_cache_weights(cache(A), b, q, 4, FAKE, 1, 0.1, 1.0, 0, FAKE, 1024, 512, None) == -2
    assert A.attn_fp8_cache_append(cache(A), b, q, q, r, None, None, 4, None) == -2
    assert A.attn_fp8_cache_workspace_bytes(cache(A), b, 4, 0) == (-2, 0)
    evict = lambda c, b: A.attn_fp8_cache_evict(c, b, cache(A), FAKE, FAKE, 1024, 512, 64, 4, 0, FAKE, FAKE, FAKE, None)
    assert evict(cache(A, n_pages=0), batch(A)) == -1
    assert evict(cache(A, n_pages=0), batch(A, B=0)) == 0


@pytest.mark.parametrize("sm,qd", [(1e-30, 1e-30), (1e30, 1e30), (1e-20, 1e-19), (3e38, 1.0)])
def test_factors_that_fp32_does_not_hold_are_refused(A, sm, qd):
    """log2(e) sm_scale q_descale of 0, infinity or below 2^-126."""
    c, b, q = cache(A), batch(A), heads(A)
    assert A.attn_fp8_cache_fwd(c, b, q, 4, FAKE, 1, FAKE, 1, sm, qd, 0, None, 0, None) == -1
    assert A.attn_fp8_cache_weights(c, b, q, 4, FAKE, 1, sm, qd, 0, FAKE, 1024, 512, None) == -1
