"""Builds librapid.so (hand-written gfx950 kernels + C ABI) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librapid.so")
SIGNATURE = os.path.join(PKG, "_signature.so")
SOURCES = ["rapid_api.hip", "verify_attn.hip", "accept.hip", "accept_greedy.hip", "hbm_probe.hip", "lm_head.hip", "kv_cache.hip", "retrieve.hip",
           "kv_quant.hip", "attn_stream.hip", "attn_prefix.hip", "attn_window.hip", "kv_rope.hip", "quant_rows.hip", "lm_head_quant.hip"]
# packed-fp32 instructions are switched off on purpose: some of their forms have given
# wrong results on this hardware generation; plain fp32 code costs nothing here
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # keep MFMA accumulators in ordinary VGPRs: the default AGPR form made the
         # compiler shuttle ~450 registers per tile between the two files
         "-mllvm", "-amdgpu-mfma-vgpr-form=1",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


# The accept pass recomputes another workgroup's partial results when they do not arrive in time and
# must get the same bits: no implicit multiply-add contraction there (explicit fma calls only).
PER_FILE_FLAGS = {"accept.hip": ["-ffp-contract=off"]}


def _compile(src: str, extra) -> str:
    obj = os.path.join(CSRC, os.path.splitext(src)[0] + ".o")
    cmd = ["hipcc", *FLAGS, *PER_FILE_FLAGS.get(src, []), *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build_signature() -> str:
    """The binding's helper (csrc/signature.cpp), a Python module against torch's headers; no GPU code."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-I{d}" for d in (*cpp_extension.include_paths(), sysconfig.get_paths()["include"])), os.path.join(CSRC, "signature.cpp"),
           "-o", SIGNATURE, f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for signature.cpp:\n{r.stdout}\n{r.stderr}")
    return SIGNATURE


def build(verbose: bool = False, extra_flags=()) -> str:
    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        signature = ex.submit(build_signature)
        objs = list(ex.map(lambda s: _compile(s, list(extra_flags)), SOURCES))
        signature.result()
    cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True, extra_flags=sys.argv[1:])
