"""Build libcompresskv.so (the HIP kernels and the C ABI) for gfx950 with hipcc.

The library is built in-tree (paper_2606_24467_amd/lib/) so that it travels
with the source tree; nothing is installed.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIBDIR = os.path.join(HERE, "lib")
LIBNAME = "libcompresskv.so"
SOURCES = ["api.hip", "score_kernels.hip", "score_layers.hip", "onepass_score.hip",
           "select_gather_kernels.hip", "offline.hip", "decode_error.hip", "cache.hip",
           "attend.hip", "attend_fp4.hip", "attend_bf16.hip", "attend_f32.hip",
           "window_attention.hip", "window_prompt.hip"]
ARCH = "gfx950"
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++20", "-fPIC",
    # packed fp32 VALU instructions stay off in every kernel of this library
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # a * b + c is fused only where the source says so (__builtin_fmaf): the
    # rounding of the same device function then does not depend on the kernel
    # it is inlined into (a multi-layer call and per-layer calls give the same
    # bits whatever their kernels' template arguments)
    "-ffp-contract=off",
    "-Wall", "-Wno-unused-result",
]


def lib_path() -> str:
    return os.path.join(LIBDIR, LIBNAME)


def _hipcc() -> str:
    p = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(p):
        raise RuntimeError("hipcc not found: the HIP library cannot be built")
    return p


# Per-source additions.  The two-pass scoring kernels and the attention keep
# MFMA results in VGPRs, where the softmax arithmetic reads them (the single-pass kernel is
# left to the default heuristics: this compiler fails on it with the option).
# The attention kernels also go without clauses of loads.  The pass that forms them
# (SI Form memory clauses) lost live ranges of 16-byte loads whose words are used one
# by one: registers of V rows were given away before their last use, and the outputs
# were wrong.  Compiled with -mllvm -verify-machineinstrs it says so ("No live subrange
# at use", in a windowed kernel of attend_bf16.hip); without clauses the verifier finds
# nothing.  It costs no time that shows: of the 4-bit and fp32 sources, which pass the
# verifier either way, 20 calls took 0.96 to 1.02 times as long as with clauses.
_ATTEND = ["-mllvm", "-amdgpu-mfma-vgpr-form", "-mllvm", "-amdgpu-max-memory-clause=1"]
EXTRA = {
    "score_kernels.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "score_layers.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
    "attend_fp4.hip": _ATTEND, "attend_bf16.hip": _ATTEND, "attend_f32.hip": _ATTEND,
}


def _compile(src: str, obj: str) -> None:
    cmd = [_hipcc(), *FLAGS, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library; returns its path."""
    os.makedirs(LIBDIR, exist_ok=True)
    objdir = os.path.join(LIBDIR, "obj")
    os.makedirs(objdir, exist_ok=True)
    objs = [os.path.join(objdir, s.rsplit(".", 1)[0] + ".o") for s in SOURCES]
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        list(ex.map(_compile, SOURCES, objs))
    tmp = lib_path() + ".tmp"
    cmd = [_hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, lib_path())
    if verbose:
        print("built", lib_path())
    return lib_path()


if __name__ == "__main__":
    build(verbose=True)
