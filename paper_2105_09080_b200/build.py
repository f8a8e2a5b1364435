"""Build libgpga.so in-tree with nvcc for sm_100a (no torch extension machinery:
the boundary is a plain C ABI loaded with ctypes)."""
from __future__ import annotations

import os
import shutil
import subprocess
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB = PKG / "libgpga.so"
SOURCES = ["gpga_api.cu", "gpga_kernels.cu", "gpga_tile.cu", "gpga_logreg.cu", "gpga_logrun.cu", "gpga_noalloc.cu", "gpga_loss.cu", "gpga_shard.cu",
           "gpga_dropout.cu", "gpga_norm.cu", "gpga_norm_grad.cu", "gpga_embed.cu", "gpga_token_api.cu",
           "gpga_gemm.cu", "gpga_ff_forward.cu", "gpga_ff_few.cu", "gpga_ff_backward.cu", "gpga_orth.cu", "gpga_matrix_api.cu"]


def nvcc_path() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found; libgpga needs the CUDA toolkit to build")
    return cand


def needs_build() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    deps = list(CSRC.glob("*.cu")) + list(CSRC.glob("*.cuh")) + [PKG.parent / "include" / "gpga.h"]
    return any(p.stat().st_mtime > t for p in deps)


def build_library(force: bool = False, verbose: bool = False) -> Path:
    if not force and not needs_build():
        return LIB
    cmd = [nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3",
           "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-cudart", "static", "--threads", "0"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [str(CSRC / s) for s in SOURCES] + ["-o", str(LIB)]
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    import sys
    print(build_library(force=True, verbose="-v" in sys.argv))
