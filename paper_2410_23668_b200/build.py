"""Builds libkl.so (the C-ABI library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
LIB = PKG / "libkl.so"
SOURCES = [CSRC / "kl.cu", CSRC / "kl_paged.cu", CSRC / "kl_drafted.cu", CSRC / "kl_sample.cu"]
HEADERS = [CSRC / "kl_device.cuh", CSRC / "kl_attention_tc.cuh", CSRC / "kl_batched.cuh", CSRC / "kl_bloop.cuh", CSRC / "kl_paged.cuh", CSRC / "kl_paged_internal.h", CSRC / "kl_paged_common.cuh", CSRC / "kl_paged_host.h", CSRC / "kl_drafted.cuh",
           PKG.parent / "include" / "kl.h"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def needs_build() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    return any(f.stat().st_mtime > t for f in SOURCES + HEADERS)


def build_library(force: bool = False, verbose: bool = False) -> Path:
    if not force and not needs_build():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB.with_suffix(f".so.tmp{os.getpid()}")
    extra = os.environ.get("KL_NVCC_FLAGS", "").split()   # e.g. -DKL_MAX_KP=4096 for tuning experiments
    # the sources are compiled side by side and linked; no device code crosses from one to the other
    objs = [tmp.with_name(f"{f.stem}.{os.getpid()}.o") for f in SOURCES]
    jobs = [subprocess.Popen([nvcc, *NVCC_FLAGS, *extra, "-c", "-o", str(o), str(f)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                             text=True) for f, o in zip(SOURCES, objs)]
    said = [j.communicate()[0] for j in jobs]
    ok = all(j.returncode == 0 for j in jobs)
    if ok:
        res = subprocess.run([nvcc, *NVCC_FLAGS[:2], "--shared", "-o", str(tmp), *map(str, objs)], capture_output=True, text=True)
        said.append(res.stdout + res.stderr)
        ok = res.returncode == 0
    for o in objs:
        o.unlink(missing_ok=True)
    if verbose or not ok:
        sys.stderr.write("".join(said))
    if not ok:
        raise RuntimeError("nvcc failed building libkl.so")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build_library(force=True, verbose=True)
    print(LIB)
