"""Python binding of libattn_fp8.so (argument marshalling only).

The C entry points are exposed under their C names; ``fwd`` and
``p_underflow_count`` are thin conveniences that take torch tensors on the GPU,
check their dtypes and shapes, allocate outputs with torch and pass the
current torch stream; ``rope``, ``cache_append``, ``cache_fwd``, ``cache_weights``,
``cache_evict``, ``cache_bounds``, ``cache_select``, ``cache_fwd_blocks`` and ``cache_fwd_shared`` do the same for
the KV cache, through a native module.  Every step of the computation
runs in the HIP kernels; there is no fallback.  If the shared library is missing the import fails,
if the native module is, the cache calls do.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattn_fp8.so")

ATTN_MODE_FAITHFUL, ATTN_MODE_FAST, ATTN_MODE_NOCAST, ATTN_MODE_FP8QK = 0, 1, 2, 3
ATTN_ORDER_FORWARD, ATTN_ORDER_REVERSE = 0, 1
ATTN_OK, ATTN_ERR_INVALID_ARG, ATTN_ERR_UNSUPPORTED, ATTN_ERR_HIP = 0, -1, -2, -3
ATTN_ERR_SCRATCH = -4
ATTN_SCALE_DYNAMIC = 0x100
ATTN_TILE_256, ATTN_TILE_128 = 0x200, 0x400

MODES = {"faithful": ATTN_MODE_FAITHFUL, "fast": ATTN_MODE_FAST, "nocast": ATTN_MODE_NOCAST,
         "fp8qk": ATTN_MODE_FP8QK}
ORDERS = {"forward": ATTN_ORDER_FORWARD, "reverse": ATTN_ORDER_REVERSE}
SCALES = {"static": 0, "dynamic": ATTN_SCALE_DYNAMIC}
TILES = {None: 0, 256: ATTN_TILE_256, 128: ATTN_TILE_128}   # fast kernel schedule (None: automatic)

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                      "(hipcc --offload-arch=gfx950)")
_lib = ctypes.CDLL(LIB_PATH)


class _NoBinding:
    """In the place of the native module where it cannot be loaded: every cache call raises;
    the other calls do not need it."""

    def __init__(self, why):
        self._why = why

    def __getattr__(self, name):
        raise ImportError(f"the cache calls need _cache_binding.so ({self._why}); run "
                          "__graft_entry__.build() (g++, with this torch)") from self._why


try:
    from . import _cache_binding as _binding  # its symbols are the library's
except ImportError as e:
    _binding = _NoBinding(e)

_P, _I, _F, _Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_lib.attn_fp8_fwd.argtypes = [_P, _P, _P, _P, _P] + [_I] * 8 + [_F, _I, _P]
_lib.attn_fp8_fwd.restype = _I
_lib.attn_fp8_p_underflow_count.argtypes = [_P, _P, _P] + [_I] * 8 + [_F, _I, _I, _P, _P, _P, _P]
_lib.attn_fp8_p_underflow_count.restype = _I
_lib.attn_fp8_fwd_descaled.argtypes = [_P, _P, _P, _P, _P] + [_I] * 8 + [_F, _I, _F, _F, _F, _P]
_lib.attn_fp8_fwd_descaled.restype = _I
_lib.attn_fp8_p_underflow_count_descaled.argtypes = ([_P, _P, _P] + [_I] * 8 + [_F, _I, _I]
                                                     + [_F, _F, _F, _P, _P, _P, _P])
_lib.attn_fp8_p_underflow_count_descaled.restype = _I
_lib.attn_fp8_fwd_kv.argtypes = [_P] * 5 + [_I] * 9 + [_F, _I, _F, _F, _F, _P, _Z, _P]
_lib.attn_fp8_fwd_kv.restype = _I
_lib.attn_fp8_p_underflow_count_kv.argtypes = ([_P] * 3 + [_I] * 9 + [_F, _I, _I, _F, _F, _F]
                                               + [_P] * 4 + [_Z, _P])
_lib.attn_fp8_p_underflow_count_kv.restype = _I
_lib.attn_fp8_fwd_kv_noalloc.argtypes = [_P] * 5 + [_I] * 9 + [_F, _I, _F, _F, _F, _P]
_lib.attn_fp8_fwd_kv_noalloc.restype = _I
_lib.attn_fp8_kv_workspace_bytes.argtypes = [_I] * 9 + [ctypes.POINTER(_Z)]
_lib.attn_fp8_kv_workspace_bytes.restype = _I
_lib.attn_fp8_block_gap_diag.argtypes = ([_P, _P, _P] + [_I] * 8 + [_F, _I, _I, _F, _F, _F, _I]
                                         + [_P] * 5 + [_P])
_lib.attn_fp8_block_gap_diag.restype = _I
_lib.attn_fp8_strerror.argtypes = [_I]
_lib.attn_fp8_strerror.restype = ctypes.c_char_p
_lib.attn_fp8_version.argtypes = []
_lib.attn_fp8_version.restype = _I


class AttnError(RuntimeError):
    def __init__(self, status: int):
        super().__init__(f"attn_fp8 status {status}: {attn_fp8_strerror(status)}")
        self.status = status


# ---- the C entry points, same names, raw pointers (ints) and sizes ----

def attn_fp8_fwd(q, k, v, out, lse, B, Hq, Hkv, N, d, causal, block_kv, order, S, mode, stream):
    return _lib.attn_fp8_fwd(q, k, v, out, lse, B, Hq, Hkv, N, d, causal, block_kv, order,
                             float(S), mode, stream)


def attn_fp8_p_underflow_count(q, k, v, B, Hq, Hkv, N, d, causal, block_kv, order, S, mode,
                               n_sink, counts, out, lse, stream):
    return _lib.attn_fp8_p_underflow_count(q, k, v, B, Hq, Hkv, N, d, causal, block_kv, order,
                                           float(S), mode, n_sink, counts, out, lse, stream)


def attn_fp8_fwd_descaled(q, k, v, out, lse, B, Hq, Hkv, N, d, causal, block_kv, order, S, mode,
                          q_descale, k_descale, v_descale, stream):
    return _lib.attn_fp8_fwd_descaled(q, k, v, out, lse, B, Hq, Hkv, N, d, causal, block_kv,
                                      order, float(S), mode, float(q_descale), float(k_descale),
                                      float(v_descale), stream)


def attn_fp8_p_underflow_count_descaled(q, k, v, B, Hq, Hkv, N, d, causal, block_kv, order, S,
                                        mode, n_sink, q_descale, k_descale, v_descale, counts,
                                        out, lse, stream):
    return _lib.attn_fp8_p_underflow_count_descaled(q, k, v, B, Hq, Hkv, N, d, causal, block_kv,
                                                    order, float(S), mode, n_sink,
                                                    float(q_descale), float(k_descale),
                                                    float(v_descale), counts, out, lse, stream)


def attn_fp8_fwd_kv(q, k, v, out, lse, B, Hq, Hkv, Nq, Nk, d, causal, block_kv, order, S, mode,
                    q_descale, k_descale, v_descale, workspace, workspace_bytes, stream):
    return _lib.attn_fp8_fwd_kv(q, k, v, out, lse, B, Hq, Hkv, Nq, Nk, d, causal, block_kv, order,
                                float(S), mode, float(q_descale), float(k_descale),
                                float(v_descale), workspace, workspace_bytes, stream)


def attn_fp8_fwd_kv_noalloc(q, k, v, out, lse, B, Hq, Hkv, Nq, Nk, d, causal, block_kv, order, S,
                            mode, q_descale, k_descale, v_descale, stream):
    return _lib.attn_fp8_fwd_kv_noalloc(q, k, v, out, lse, B, Hq, Hkv, Nq, Nk, d, causal,
                                        block_kv, order, float(S), mode, float(q_descale),
                                        float(k_descale), float(v_descale), stream)


def attn_fp8_p_underflow_count_kv(q, k, v, B, Hq, Hkv, Nq, Nk, d, causal, block_kv, order, S,
                                  mode, n_sink, q_descale, k_descale, v_descale, counts, out,
                                  lse, workspace, workspace_bytes, stream):
    return _lib.attn_fp8_p_underflow_count_kv(q, k, v, B, Hq, Hkv, Nq, Nk, d, causal, block_kv,
                                              order, float(S), mode, n_sink, float(q_descale),
                                              float(k_descale), float(v_descale), counts, out,
                                              lse, workspace, workspace_bytes, stream)


def attn_fp8_kv_workspace_bytes(B, Hq, Hkv, Nq, Nk, d, causal, block_kv, mode):
    """Returns (status, bytes)."""
    n = _Z(0)
    st = _lib.attn_fp8_kv_workspace_bytes(B, Hq, Hkv, Nq, Nk, d, causal, block_kv, mode,
                                          ctypes.byref(n))
    return st, n.value


def attn_fp8_block_gap_diag(q, k, v, B, Hq, Hkv, N, d, causal, block_kv, order, S, mode, n_sink,
                            q_descale, k_descale, v_descale, nbins, gap_hist, blk_zero, counts,
                            out, lse, stream):
    return _lib.attn_fp8_block_gap_diag(q, k, v, B, Hq, Hkv, N, d, causal, block_kv, order,
                                        float(S), mode, n_sink, float(q_descale),
                                        float(k_descale), float(v_descale), nbins, gap_hist,
                                        blk_zero, counts, out, lse, stream)


def attn_fp8_strerror(status: int) -> str:
    return _lib.attn_fp8_strerror(status).decode()


def attn_fp8_version() -> int:
    return _lib.attn_fp8_version()


# ---- the KV cache (include/attn_fp8_cache.h): structures and C entry points ----

ATTN_TYPE_F32, ATTN_TYPE_BF16, ATTN_TYPE_F16, ATTN_TYPE_E4M3 = 0, 1, 2, 3
ATTN_ROPE_HALF, ATTN_ROPE_INTERLEAVED = 0, 1

LAYOUTS = {"half": ATTN_ROPE_HALF, "interleaved": ATTN_ROPE_INTERLEAVED}


class attn_fp8_cache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_scale", _P), ("v_scale", _P), ("n_pages", _I), ("Hkv", _I),
                ("page", _I), ("d", _I)]


class attn_fp8_batch(ctypes.Structure):
    _fields_ = [("pages", _P), ("lens", _P), ("cu", _P), ("B", _I), ("W", _I), ("T", _I), ("max_q", _I)]


class attn_fp8_heads(ctypes.Structure):
    _fields_ = [("data", _P), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("type", _I)]


class attn_fp8_rotation(ctypes.Structure):
    _fields_ = [("table", _P), ("positions", _P), ("n_pos", _I), ("rot", _I), ("layout", _I)]


_L = ctypes.c_int64
_PC, _PB, _PH, _PR = (ctypes.POINTER(t) for t in (attn_fp8_cache, attn_fp8_batch, attn_fp8_heads,
                                                  attn_fp8_rotation))
_lib.attn_fp8_rope.argtypes = [_PH, _PH, _I, _I, _I, _PR, _P]
_lib.attn_fp8_rope.restype = _I
_lib.attn_fp8_cache_append.argtypes = [_PC, _PB, _PH, _PH, _PR, _PH, _PH, _I, _P]
_lib.attn_fp8_cache_append.restype = _I
_lib.attn_fp8_cache_fwd.argtypes = [_PC, _PB, _PH, _I, _P, _I, _P, _I, _F, _F, _I, _P, _Z, _P]
_lib.attn_fp8_cache_fwd.restype = _I
_lib.attn_fp8_cache_workspace_bytes.argtypes = [_PC, _PB, _I, _I, ctypes.POINTER(_Z)]
_lib.attn_fp8_cache_workspace_bytes.restype = _I
_lib.attn_fp8_cache_weights.argtypes = [_PC, _PB, _PH, _I, _P, _I, _F, _F, _I, _P, _L, _L, _P]
_lib.attn_fp8_cache_weights.restype = _I
_lib.attn_fp8_cache_evict.argtypes = [_PC, _PB, _PC, _P, _P, _L, _L, _I, _I, _I, _P, _P, _P, _P]
_lib.attn_fp8_cache_evict.restype = _I
# include/attn_fp8_parts.h
_lib.attn_fp8_cache_bounds.argtypes = [_PC, _PB, _P, _P]
_lib.attn_fp8_cache_bounds.restype = _I
_lib.attn_fp8_cache_select.argtypes = [_PC, _PB, _PH, _I, _P, _P] + [_I] * 6 + [_P, _Z, _P]
_lib.attn_fp8_cache_select.restype = _I
_lib.attn_fp8_cache_select_workspace_bytes.argtypes = [_PC, _PB, _I, _I, _I, _I, ctypes.POINTER(_Z)]
_lib.attn_fp8_cache_select_workspace_bytes.restype = _I
_lib.attn_fp8_cache_fwd_blocks.argtypes = [_PC, _PB, _PH, _I, _P, _I, _I, _P, _I, _P, _I, _F, _F, _P, _Z, _P]
_lib.attn_fp8_cache_fwd_blocks.restype = _I
_lib.attn_fp8_cache_blocks_workspace_bytes.argtypes = [_PC, _PB, _I, _I, _I, ctypes.POINTER(_Z)]
_lib.attn_fp8_cache_blocks_workspace_bytes.restype = _I
_lib.attn_fp8_cache_fwd_shared.argtypes = [_PC, _PB, _I, _PH, _I, _P, _I, _P, _I, _F, _F, _I, _P, _Z, _P]
_lib.attn_fp8_cache_fwd_shared.restype = _I
_lib.attn_fp8_cache_shared_workspace_bytes.argtypes = [_PC, _PB, _I, _I, _I, ctypes.POINTER(_Z)]
_lib.attn_fp8_cache_shared_workspace_bytes.restype = _I

attn_fp8_rope = _lib.attn_fp8_rope
attn_fp8_cache_append = _lib.attn_fp8_cache_append
attn_fp8_cache_fwd = _lib.attn_fp8_cache_fwd
attn_fp8_cache_weights = _lib.attn_fp8_cache_weights
attn_fp8_cache_evict = _lib.attn_fp8_cache_evict
attn_fp8_cache_bounds = _lib.attn_fp8_cache_bounds
attn_fp8_cache_select = _lib.attn_fp8_cache_select
attn_fp8_cache_fwd_blocks = _lib.attn_fp8_cache_fwd_blocks
attn_fp8_cache_fwd_shared = _lib.attn_fp8_cache_fwd_shared


def attn_fp8_cache_workspace_bytes(cache, batch, Hq, max_len):
    """Returns (status, bytes)."""
    n = _Z(0)
    st = _lib.attn_fp8_cache_workspace_bytes(cache, batch, Hq, max_len, ctypes.byref(n))
    return st, n.value


def attn_fp8_cache_select_workspace_bytes(cache, batch, Hq, take, run, max_len):
    """Returns (status, bytes)."""
    n = _Z(0)
    st = _lib.attn_fp8_cache_select_workspace_bytes(cache, batch, Hq, take, run, max_len, ctypes.byref(n))
    return st, n.value


def attn_fp8_cache_blocks_workspace_bytes(cache, batch, Hq, take, run):
    """Returns (status, bytes)."""
    n = _Z(0)
    st = _lib.attn_fp8_cache_blocks_workspace_bytes(cache, batch, Hq, take, run, ctypes.byref(n))
    return st, n.value


def attn_fp8_cache_shared_workspace_bytes(cache, batch, shared, Hq, max_len):
    """Returns (status, bytes)."""
    n = _Z(0)
    st = _lib.attn_fp8_cache_shared_workspace_bytes(cache, batch, shared, Hq, max_len, ctypes.byref(n))
    return st, n.value


# ---- torch conveniences ----

_FAST_QK = (torch.bfloat16, torch.int16, torch.uint16)
_FAST_V = (torch.float8_e4m3fn, torch.uint8)


def _check(q, k, v, mode):
    qs, ks, vs = q.shape, k.shape, v.shape
    if len(qs) != 4 or len(ks) != 4 or len(vs) != 4:
        raise ValueError("q, k, v must be [B, H, N, d]")
    B, Hq, N, d = qs
    Bk, Hkv, Nk, dk = ks
    if ks != vs or Bk != B or Nk < N or dk != d:
        raise ValueError(f"shape mismatch: q {tuple(qs)} k {tuple(ks)} v {tuple(vs)}")
    if not (q.is_cuda and k.is_cuda and v.is_cuda and q.is_contiguous() and k.is_contiguous()
            and v.is_contiguous()):
        raise ValueError("q, k, v must be contiguous device tensors")
    if mode == ATTN_MODE_FAST:
        if q.dtype not in _FAST_QK or k.dtype not in _FAST_QK or v.dtype not in _FAST_V:
            raise TypeError("fast mode takes bfloat16 q/k and float8_e4m3fn (or uint8) v")
    elif mode == ATTN_MODE_FP8QK:
        if q.dtype not in _FAST_V or k.dtype not in _FAST_V or v.dtype not in _FAST_V:
            raise TypeError("fp8qk mode takes float8_e4m3fn (or uint8) q, k and v")
    elif q.dtype != torch.float32 or k.dtype != torch.float32 or v.dtype != torch.float32:
        raise TypeError("faithful / nocast modes take float32 q, k, v")
    return B, Hq, Hkv, N, d, Nk


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle without a Stream object around it: 0.1 us against
# 2.9 (a short call's host time is 16 us in all)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None and _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


@functools.lru_cache(maxsize=4096)
def _kv_workspace_bytes(device_index, *shape):
    """The size depends on the shape and on the device's CU count alone."""
    st, n = attn_fp8_kv_workspace_bytes(*shape)
    if st != ATTN_OK:
        raise AttnError(st)
    return n


def kv_workspace(B, Hq, Hkv, N, Nk, d, causal, block_kv, mode, device, stream=None):
    """A device workspace (torch-allocated) for a KV-cache call of this shape,
    or None when the call does not split.  stream: the stream the call runs on,
    if not the current one; the memory belongs to it, so that torch hands it out
    again only in that stream's order."""
    n = _kv_workspace_bytes(torch.cuda.current_device(), B, Hq, Hkv, N, Nk, d, int(bool(causal)),
                            int(block_kv), mode)
    if not n:
        return None
    if stream is None:
        return torch.empty(n, dtype=torch.uint8, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(n, dtype=torch.uint8, device=device)


def fwd(q, k, v, *, S: float = 256.0, order: str = "reverse", causal: bool = False,
        block_kv: int = 128, mode: str = "fast", out=None, lse=None, want_lse: bool = True,
        stream=None, scale: str = "static", descales=(1.0, 1.0, 1.0), tile=None):
    """Attention forward; returns (out [B,Hq,N,d] float32, lse [B,Hq,N] float32 or None).
    k, v may hold more keys than q has rows (a KV cache): query row r then
    sits at key position Nk - N + r; the call's workspace, if it splits, is
    taken from torch's allocator on q's device.
    scale="dynamic" ORs ATTN_SCALE_DYNAMIC into the mode (S = 2^k0, k0 <= 8);
    descales = per-tensor (q, k, v) descales of the stored values; tile = 256 or
    128 forces the fast kernel's schedule (ATTN_TILE_*), None lets the library pick."""
    m = MODES[mode]
    B, Hq, Hkv, N, d, Nk = _check(q, k, v, m)
    if out is None:
        out = torch.empty((B, Hq, N, d), dtype=torch.float32, device=q.device)
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, N), dtype=torch.float32, device=q.device)
    ws = kv_workspace(B, Hq, Hkv, N, Nk, d, causal, block_kv, m, q.device, stream) if Nk != N else None
    st = attn_fp8_fwd_kv(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, Hq, Hkv, N, Nk, d,
                         int(bool(causal)), int(block_kv), ORDERS[order], S,
                         m | SCALES[scale] | TILES[tile], *descales, _ptr(ws),
                         0 if ws is None else ws.numel(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st)
    return out, lse


def p_underflow_count(q, k, v, *, S: float = 256.0, order: str = "reverse", causal: bool = False,
                      block_kv: int = 128, mode: str = "fast", n_sink: int = 4, out=None, lse=None,
                      stream=None, scale: str = "static", descales=(1.0, 1.0, 1.0), tile=None):
    """P-underflow diagnostic; returns counts [B,Hq,N,3] uint32 (as int32 storage)."""
    m = MODES[mode]
    B, Hq, Hkv, N, d, Nk = _check(q, k, v, m)
    counts = torch.empty((B, Hq, N, 3), dtype=torch.int32, device=q.device)
    ws = kv_workspace(B, Hq, Hkv, N, Nk, d, causal, block_kv, m, q.device, stream) if Nk != N else None
    st = attn_fp8_p_underflow_count_kv(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, N, Nk, d,
                                       int(bool(causal)), int(block_kv), ORDERS[order], S,
                                       m | SCALES[scale] | TILES[tile], int(n_sink), *descales,
                                       _ptr(counts),
                                       _ptr(out), _ptr(lse), _ptr(ws),
                                       0 if ws is None else ws.numel(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st)
    return counts


def block_gap_diag(q, k, v, *, S: float = 256.0, order: str = "reverse", causal: bool = False,
                   block_kv: int = 128, mode: str = "fast", n_sink: int = 4, nbins: int = 32,
                   stream=None, scale: str = "static", descales=(1.0, 1.0, 1.0), tile=None):
    """Per-block diagnostic; returns (gap_hist [B,Hq,nblk,nbins], blk_zero [B,Hq,nblk],
    counts [B,Hq,N,3]), all uint32 held in int32 storage."""
    m = MODES[mode]
    B, Hq, Hkv, N, d, Nk = _check(q, k, v, m)
    if Nk != N:
        raise ValueError("block_gap_diag takes square problems (as many keys as query rows)")
    nblk = (N + block_kv - 1) // block_kv
    hist = torch.empty((B, Hq, nblk, nbins), dtype=torch.int32, device=q.device)
    bz = torch.empty((B, Hq, nblk), dtype=torch.int32, device=q.device)
    counts = torch.empty((B, Hq, N, 3), dtype=torch.int32, device=q.device)
    st = attn_fp8_block_gap_diag(_ptr(q), _ptr(k), _ptr(v), B, Hq, Hkv, N, d, int(bool(causal)),
                                 int(block_kv), ORDERS[order], S, m | SCALES[scale] | TILES[tile],
                                 int(n_sink),
                                 *descales, int(nbins), _ptr(hist), _ptr(bz), _ptr(counts), None,
                                 None, _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st)
    return hist, bz, counts


# ---- the KV cache: torch conveniences (csrc/cache_binding.cpp checks the tensors, allocates
# outputs and workspaces and passes the current stream) ----

_OUT_TYPES = {torch.float32: ATTN_TYPE_F32, torch.bfloat16: ATTN_TYPE_BF16}


class KVCache(NamedTuple):
    """An E4M3 cache in pages: k, v [pages, Hkv, page, d] float8_e4m3fn (or uint8),
    k_scale, v_scale [pages, Hkv] uint8; a code stands for code * 2^(byte - 127)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor


def kv_cache(n_pages, Hkv, d, *, page: int = 128, device="cuda"):
    """A KVCache of empty (zero) pages."""
    def codes():
        return torch.zeros((n_pages, Hkv, page, d), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)

    def scales():
        return torch.zeros((n_pages, Hkv), dtype=torch.uint8, device=device)

    return KVCache(codes(), codes(), scales(), scales())


def _call(stream, f, *args):
    """A call of the native binding, on `stream` (outputs and workspace belong to it) or
    the current one."""
    if stream is None:
        r = f(*args)
    else:
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream.cuda_stream)
        with torch.cuda.stream(stream):
            r = f(*args)
    if type(r) is int:
        raise AttnError(r)
    return r


def rope_table(n_pos, rot, *, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
               original: int = 0, ramp=(1.0, 32.0), device="cuda"):
    """cos and sin of the rotations, float32 [n_pos, rot / 2, 2], computed in 64 bits
    and rounded once: pair i turns by p * base^(-2 i / rot) at position p.  Scaled
    for contexts `factor` times longer than the model was trained on:
      "linear"  positions are divided by factor;
      "base"    the base grows to base * factor^(rot / (rot - 2)), which divides the
                slowest pair's angle by factor and leaves the fastest one's;
      "ramp"    a pair that makes fewer than ramp[0] turns over the `original`
                positions is divided by factor, one of more than ramp[1] turns is
                left, those between are blended linearly in the number of turns."""
    if rot < 2 or rot % 2 or n_pos < 1 or factor <= 0 or base <= 0:
        raise ValueError("rope_table needs n_pos >= 1, an even rot >= 2, and positive base and factor")
    i = torch.arange(rot // 2, dtype=torch.float64, device=device)
    if scaling == "base":
        if rot < 4:
            raise ValueError("scaling by the base needs rot >= 4")
        base = base * factor ** (rot / (rot - 2))
    freq = base ** (-2.0 * i / rot)
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "ramp":
        lo, hi = ramp
        if original < 1 or not 0 <= lo < hi:
            raise ValueError("scaling by a ramp needs original >= 1 and 0 <= ramp[0] < ramp[1]")
        keep = ((original * freq / (2 * math.pi) - lo) / (hi - lo)).clamp(0.0, 1.0)
        freq = freq * keep + freq / factor * (1 - keep)
    elif scaling not in ("none", "base"):
        raise ValueError(f"unknown scaling {scaling!r}")
    angle = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * freq
    return torch.stack((torch.cos(angle), torch.sin(angle)), -1).float().contiguous()


def rope(x, table, positions, *, layout: str = "half", out=None, stream=None):
    """Rotary positions: x [T, H, d] (float32, bfloat16 or float16, any strides of tokens
    and heads that are multiples of 16 bytes) with its first rot channels rotated by
    row positions[t] of the table (rope_table); layout "half" pairs channel i with
    i + rot / 2, "interleaved" 2 i with 2 i + 1.  out may be x."""
    return _call(stream, _binding.rope, x, table, positions, LAYOUTS[layout], out)


def cache_append(cache, k, v, pages, lens, *, cu=None, max_q=None, table=None, positions=None,
                 layout: str = "half", q=None, q_out=None, stream=None):
    """Writes new tokens k, v [T, Hkv, d] into the pages of their sequences: k rotated
    (with a table), both rounded to E4M3 on the scale of their block.  pages int32
    [B, W], lens int32 [B] (the new tokens included), cu int32 [B + 1] with max_q (None:
    T / B tokens each).  positions None: the tokens' places in their sequences.  With
    q [T, Hq, d] its rotation is done in the same launch and returned, in q's type: cache_fwd
    takes bfloat16 (or float8_e4m3fn), so float32 and float16 ones are converted between.
    Rows of the returned q that belong to no sequence's first max_q tokens are left unset."""
    return _call(stream, _binding.append, cache, k, v, pages, lens, cu, max_q, table, positions, LAYOUTS[layout], q,
                 q_out)


def cache_fwd(q, cache, pages, lens, *, cu=None, max_q=None, causal: bool = True, sm_scale=None,
              q_descale: float = 1.0, max_len: int = 0, out=None, out_dtype=torch.bfloat16, lse=None,
              want_lse: bool = True, stream=None):
    """Attention of new tokens q [T, Hq, d] (bfloat16 or float8_e4m3fn) over their
    sequences' cached ones, the new ones included; returns (out [T, Hq, d] of out_dtype
    (bfloat16 or float32), lse [T, Hq] float32 or None).  Token i of a sequence's n is
    at position lens[b] - n + i and sees the keys up to it (causal=False: all); before
    position 0, as the front of a padded batch, it sees none and gets out = 0, lse = -inf.
    pages, lens, cu, max_q as for cache_append.  sm_scale None: 1 / sqrt(d).
    max_len: no sequence is longer (0: as long as pages allows).  Rows that belong to no
    sequence's first max_q tokens (behind cu[B], say) are not written: in outputs that the
    call allocates they hold anything."""
    return _call(stream, _binding.fwd, q, cache, pages, lens, cu, max_q, causal, sm_scale, q_descale, max_len, out,
                 _OUT_TYPES[out_dtype], lse, want_lse)


def cache_weights(q, lse, cache, pages, lens, weights, *, cu=None, max_q=None, causal: bool = True, sm_scale=None,
                  q_descale: float = 1.0, max_len: int = 0, stream=None):
    """Adds to weights [B, Hkv, n] (float32, in place; n at least the longest sequence,
    max_len or W * page) the attention weight that each cached token receives from the
    new tokens q and the query heads of its group; lse is cache_fwd's for the same call."""
    return _call(stream, _binding.weights, q, lse, cache, pages, lens, weights, cu, max_q, causal, sm_scale, q_descale,
                 max_len)


def cache_evict(cache, pages, lens, weights, to, new_pages, budget, *, n_sink: int = 4, n_recent: int = 0,
                kept=None, new_lens=None, new_weights=None, stream=None):
    """Moves the `budget` tokens of every sequence and KV head that matter most into the
    pages new_pages int32 [B, ceil(budget / page)] of the cache `to` (which may be
    `cache`, then pages that hold none of these sequences): the first n_sink, the last
    n_recent, and the ones of the largest weights [B, Hkv, n] (equal ones: the earlier).
    Returns (kept [B, Hkv, budget] int32: where each was, then -1; new_lens [B] int32;
    new_weights [B, Hkv, budget] float32: theirs, then 0); given ones overlap no input."""
    return _call(stream, _binding.evict, cache, pages, lens, weights, to, new_pages, budget, n_sink, n_recent, kept,
                 new_lens, new_weights)


# ---- attention over parts of the cache ----

def key_bounds(n_pages, Hkv, d, *, device="cuda"):
    """Room for the bounds of a cache's keys, float8_e4m3fn [pages, Hkv, 2, d] of zeros: the
    least code of each channel of a page, and the largest."""
    return torch.zeros((n_pages, Hkv, 2, d), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)


def cache_bounds(cache, pages, lens, bounds, *, cu=None, max_q=None, stream=None):
    """Writes the bounds (key_bounds) of the pages that hold the last max_q tokens of each
    sequence (None: all of them), or with cu int32 [B + 1] the last cu[b + 1] - cu[b], of which the
    first max_q count, as cache_append has written them; returns bounds.  To be called after each
    append: a page's codes change when its scale grows."""
    return _call(stream, _binding.bounds, cache, pages, lens, bounds, cu, max_q)


def cache_select(q, cache, pages, lens, bounds, take, *, cu=None, max_q=None, run: int = 1, n_first: int = 1,
                 n_last: int = 1, causal: bool = True, max_len: int = 0, blocks=None, stream=None):
    """The `take` pages of each run of `run` new tokens and KV head whose bounds allow the largest
    scores of the run's queries, as places in the sequence's row of pages: int32
    [B, ceil(max_q / run), Hkv, take], ascending, then -1.  The first n_first and the last n_last
    of the pages that the run sees are always among them; equal scores: the earlier page.  Runs of
    more than one token may cross the end of a page: all of them keep their own page, and so see
    themselves, with n_last = 1 + ceil((run - 1) / page).  q and the others as for cache_fwd."""
    return _call(stream, _binding.select, q, cache, pages, lens, bounds, take, cu, max_q, run, n_first, n_last, causal,
                 max_len, blocks)


def cache_fwd_blocks(q, cache, pages, lens, blocks, *, cu=None, max_q=None, run: int = 1, causal: bool = True,
                     sm_scale=None, q_descale: float = 1.0, out=None, out_dtype=torch.bfloat16, lse=None,
                     want_lse: bool = True, stream=None):
    """cache_fwd over the pages of lists alone: blocks int32 [B, ceil(max_q / run), Hkv, take], one
    list for each run of `run` new tokens and KV head, as cache_select gives them (any order; below
    0: none; a page listed twice counts twice).  A query sees of them what it sees of the sequence."""
    return _call(stream, _binding.fwd_blocks, q, cache, pages, lens, blocks, cu, max_q, run, causal, sm_scale, q_descale,
                 out, _OUT_TYPES[out_dtype], lse, want_lse)


def cache_fwd_shared(q, cache, pages, lens, n_shared, *, cu=None, max_q=None, causal: bool = True, sm_scale=None,
                     q_descale: float = 1.0, max_len: int = 0, out=None, out_dtype=torch.bfloat16, lse=None,
                     want_lse: bool = True, stream=None):
    """cache_fwd for sequences that begin with the same n_shared pages (those of the first row of
    pages; the other rows' first n_shared entries are not looked at): the same result, with these
    pages read once for the queries of all sequences (a few short ones: cache_fwd is faster)."""
    return _call(stream, _binding.fwd_shared, q, cache, pages, lens, n_shared, cu, max_q, causal, sm_scale, q_descale,
                 max_len, out, _OUT_TYPES[out_dtype], lse, want_lse)
