"""Builds libjb.so (the CUDA kernels and the C ABI) in-tree for sm_103a.

    python -m paper_2306_10015_gb300.build

Translation units compiled in parallel by nvcc, linked with the static
CUDA runtime. No fast-math: the fp32 arithmetic of the kernels is written with
explicit round-to-nearest intrinsics and must not be re-associated.
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(OUT_DIR, "libjb.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
SOURCES = ["jb_kernels.cu", "jb_q4.cu", "jb_attend.cu", "jb_pages.cu", "jb_sample.cu", "jb_capi.cpp",
           "jb_answer_capi.cpp", "jb_append.cu", "jb_keep.cu", "jb_tree.cu", "jb_tree_bf16.cu", "jb_q4_matmul.cu", "jb_q4_tiles.cu", "jb_draft_capi.cpp"]
HEADERS = ["jb_rng.cuh", "jb_internal.h", "jb_offgrid.h", "jb_answer.h", "jb_host.h", "jb_launch.cuh",
           "jb_check.h", "jb_draft.h", "jb_scores.cuh", "jb_tree.cuh", "jb_tcgen05.cuh", "jb_tensor_map.h", "jb_q4_halves.cuh"]


def nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(INCLUDE, "jb.h"),
                                                                  os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile libjb.so if any source is newer than it; returns its path."""
    if not force and not _stale():
        return LIB
    os.makedirs(OUT_DIR, exist_ok=True)
    # no implicit a * b + c -> fma contraction on either side: every rounding in
    # the device code is the one its intrinsic names
    common = ARCH + ["-O3", "-std=c++17", "-lineinfo", "-I", INCLUDE, "-I", CSRC,
                     "--fmad=false", "-Xcompiler", "-fPIC,-fvisibility=hidden,-ffp-contract=off",
                     "--expt-relaxed-constexpr"]
    if verbose:
        common += ["-Xptxas", "-v"]
    procs, objs = [], []
    for src in SOURCES:
        obj = os.path.join(OUT_DIR, os.path.splitext(src)[0] + ".o")
        objs.append(obj)
        cmd = [nvcc()] + common + ["-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for cmd, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out.decode(errors="replace"))
        if p.returncode != 0:
            failed.append(" ".join(cmd))
    if failed:
        raise RuntimeError("nvcc failed:\n" + "\n".join(failed))
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.run([nvcc()] + ARCH + ["-shared", "-cudart", "static", "-o", tmp] + objs, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv, verbose="-v" in sys.argv)
    print(LIB)
