"""Build libattn_fp8.so (the HIP kernels and the C ABI) for gfx950 with hipcc, and
_cache_binding.so (the cache calls on torch tensors) with g++.

Every call compiles from source.  Objects go to ``_build/`` at the repository
root; the shared libraries land next to this file so they travel with the tree.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libattn_fp8.so")
BINDING = os.path.join(HERE, "_cache_binding.so")

SOURCES = ["attn_fp8_abi.hip", "attn_fast.hip", "attn_fast_pair.hip", "attn_fast_qk8.hip",
           "attn_fast_qk8_pair.hip", "attn_faithful.hip", "attn_prefill.hip", "attn_kv_bf16_16.hip",
           "attn_kv_bf16_32.hip", "attn_kv_qk8_16.hip", "attn_kv_qk8_32.hip", "cache_abi.hip",
           "cache_rope.hip", "cache_fwd.hip", "cache_weights.hip", "cache_evict.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# -packed-fp32-ops: no packed FP32 VALU instructions anywhere in the device code
HIP_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Wno-unused-command-line-argument"]


def _compile(src: str, obj: str) -> None:
    cmd = [HIPCC, *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")


def hip_library(jobs: int | None = None) -> str:
    os.makedirs(BUILD, exist_ok=True)
    objs = [os.path.join(BUILD, s.replace(".hip", ".o")) for s in SOURCES]
    jobs = jobs or min(len(SOURCES), max(1, (os.cpu_count() or 2)))
    with cf.ThreadPoolExecutor(jobs) as ex:
        list(ex.map(lambda so: _compile(*so), zip(SOURCES, objs)))
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


def binding() -> str:
    """The Python module of the cache calls; links the library and torch."""
    import sysconfig

    from torch.utils import cpp_extension

    include = [*cpp_extension.include_paths(), sysconfig.get_paths()["include"], "/opt/rocm/include"]
    tmp = BINDING + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM",
           *("-I" + d for d in include), os.path.join(CSRC, "cache_binding.cpp"), "-o", tmp,
           *("-L" + d for d in cpp_extension.library_paths()), "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10",
           "-lc10_hip", "-L" + HERE, "-lattn_fp8", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for cache_binding.cpp:\n{r.stderr}")
    os.replace(tmp, BINDING)
    return BINDING


if __name__ == "__main__":
    print(hip_library())
    print(binding())
    sys.exit(0)
