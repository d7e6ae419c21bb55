"""Compile the CUDA sources of this package into libaero_b200.so (sm_100a only).

Usage: python -m paper_2602_14338_b200.build   (needs nvcc on PATH or in /usr/local/cuda/bin)
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libaero_b200.so")
SOURCES = ["api.cu", "group_stage.cu", "loss_common.cu", "loss_fp32.cu", "loss_fwd_tc.cu", "loss_bwd_tc.cu", "step_host.cu", "alloc_sim.cu", "step_fused_tc.cu", "selftest.cu",
           "rmsnorm.cu", "embed.cu", "lmhead_q8.cu", "distill.cu"]
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return exe


def _stale() -> bool:
    if not os.path.exists(OUT):
        return True
    t = os.path.getmtime(OUT)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "aero.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False, out: str | None = None, defines=()) -> str:
    """Build the library.  `out` and `defines` (e.g. ["AERO_LMHEAD_STAGES=3"]) make a tuning variant
    somewhere else; binding.py loads it when AERO_B200_LIB names it."""
    if out is None and not force and not _stale():
        return OUT
    nvcc = _nvcc()
    objdir = os.path.join(HERE, "_build" if out is None else "_build_" + "_".join(defines).replace("=", ""))
    os.makedirs(objdir, exist_ok=True)

    def compile_one(src: str) -> str:
        obj = os.path.join(objdir, src.replace(".cu", ".o"))
        cmd = [nvcc, *FLAGS, *[f"-D{d}" for d in defines], "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    target = out or OUT
    r = subprocess.run([nvcc, "-shared", "-o", target, *objs, "-gencode", "arch=compute_100a,code=sm_100a"],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    return target


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
