"""The library's plan of a cache attention call and its choice of an eviction's kernel (host code;
no GPU needed), so that a test can say which kernel it runs."""
from __future__ import annotations

import ctypes

from paper_2606_06521_amd import attn_fp8


class Plan(ctypes.Structure):
    """attn::FwdPlan"""
    _fields_ = [("rows", ctypes.c_int), ("tiles", ctypes.c_int), ("chunk", ctypes.c_int),
                ("ranges", ctypes.c_int), ("bytes", ctypes.c_size_t)]


_fn = ctypes.CDLL(attn_fp8.LIB_PATH)["_ZN4attn14cache_fwd_planEiiiiiii"]
_fn.argtypes, _fn.restype = [ctypes.c_int] * 7, Plan


def fwd_plan(B, Hkv, G, max_q, max_len, d, n_cu=256):
    """rows: 16 or 128 query rows per tile; ranges: parts of the keys, 1 unless split."""
    return _fn(B, Hkv, G, max_q, max_len, d, n_cu)


def max_q_of_tall_tiles(B, Hkv, G, at_least, max_len, d, n_cu=256):
    """A bound on the new tokens, at least `at_least`, with which a call runs on 128-row tiles."""
    q = at_least
    while fwd_plan(B, Hkv, G, q, max_len, d, n_cu).rows != 128:
        q *= 2
        assert q * G <= 1 << 20, (B, Hkv, G, at_least, max_len, d)
    return q
