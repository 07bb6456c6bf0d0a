"""Build libsift.so (the HIP kernels and the C ABI) for gfx950, in-tree.

    python -m paper_2606_09441_amd.build

Every source is compiled by hipcc for gfx950 only; packed-FP32 instructions
are disabled (ordinary float code is generated instead).
"""

from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_PATH = os.path.join(HERE, "libsift.so")
BUILD_DIR = os.path.join(ROOT, "_build")

SOURCES = ["decode.hip", "attn_bf16.hip", "attn_f32.hip", "attn_dense.hip", "cache_attn.hip", "cache_wide.hip",
           "cache_append.hip", "cache_codes.hip", "codes_wide.hip", "cache_weights.hip", "cache_evict.hip", "extract.hip", "rope.hip",
           "rotary.hip", "layer_ops.hip", "sift_api.cpp",
           "extract_api.cpp", "layer_api.cpp", "cache_api.cpp"]
# Per-source extra flags.  The bf16 attention kernel takes row maxima of MFMA
# results that are finite or -inf (masked): NaN canonicalisation around
# fmaxf would only add instructions, so NaNs are not honoured there.
EXTRA = {"attn_bf16.hip": ["-fno-honor-nans"], "extract.hip": ["-fno-honor-nans"]}

ARCH = "gfx950"
COMMON = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-fPIC",
    "-std=c++17",
    "-Wall",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE,
    "-I", CSRC,
]


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build libsift)")


def _compile(src: str, hipcc: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = [hipcc, *COMMON, *EXTRA.get(src, [])]
    if src.endswith(".cpp"):
        cmd += ["-x", "hip"]
    cmd += ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = [ln for ln in (r.stdout + r.stderr).splitlines()
            if "packed-fp32-ops" not in ln]   # the host pass does not know the feature
    if r.returncode != 0:
        raise RuntimeError(f"compiling {src} failed:\n" + "\n".join(msgs))
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source and link LIB_PATH; returns its path."""
    hipcc = _hipcc()
    os.makedirs(BUILD_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, hipcc), SOURCES))
    tmp = LIB_PATH + ".tmp"
    cmd = [hipcc, f"--offload-arch={ARCH}", "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("linking libsift.so failed:\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB_PATH)
    if verbose:
        print(f"built {LIB_PATH}")
    return LIB_PATH


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
