"""Build step of the Forcing-KV library: compiles the CUDA sources for sm_103a into
`libfk.so` next to this file (in-tree).  Translation units compile in parallel; a
unit is recompiled only when it, or a header, is newer than its object."""
from __future__ import annotations

import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libfk.so")
SOURCES = ["fk_host.cu", "fk_copy.cu", "fk_score.cu", "fk_attn.cu", "fk_quant.cu",
           "fk_paged_host.cu", "fk_paged_append.cu", "fk_paged_few.cu", "fk_paged_chunk.cu",
           "fk_rotary.cu", "fk_linear_host.cu", "fk_linear_few.cu", "fk_linear_chunk.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libfk.so")


def _headers_mtime() -> float:
    hs = [os.path.join(INCLUDE, "fk.h")] + [os.path.join(CSRC, f) for f in os.listdir(CSRC)
                                             if f.endswith(".h")]
    return max(os.path.getmtime(h) for h in hs)


def _run(cmd: list[str]) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("command failed: %s\n%s%s" % (" ".join(cmd), r.stdout, r.stderr))


def build(force: bool = False, verbose: bool = False, extra_flags: list[str] | None = None) -> str:
    """Compile (if needed) and return the path of libfk.so."""
    nvcc = _nvcc()
    os.makedirs(BUILD_DIR, exist_ok=True)
    hdr_t = _headers_mtime()
    jobs = []
    objs = []
    for src in SOURCES:
        sp = os.path.join(CSRC, src)
        op = os.path.join(BUILD_DIR, src.replace(".cu", ".o"))
        objs.append(op)
        stale = force or not os.path.exists(op) or os.path.getmtime(op) < max(os.path.getmtime(sp), hdr_t)
        if stale:
            jobs.append([nvcc] + ARCH + FLAGS + (extra_flags or []) + ["-c", sp, "-o", op])
    if jobs:
        with ThreadPoolExecutor(max_workers=len(jobs)) as ex:
            for cmd in jobs:
                if verbose:
                    print(" ".join(cmd))
            list(ex.map(_run, jobs))
    if jobs or not os.path.exists(LIB_PATH):
        tmp = LIB_PATH + ".tmp"
        _run([nvcc] + ARCH + ["-shared", "-o", tmp] + objs)
        os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
