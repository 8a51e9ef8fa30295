"""Build the scheduler library in-tree: one nvcc per translation unit (in parallel), one link.

Output: paper_2609_33224_gb300/_build/libpackserve.so, code for sm_103a only, CUDA runtime linked
statically so the library needs nothing but the driver at load time.
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
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libpackserve.so")
SOURCES = ["api.cu", "probe.cu", "score.cu", "greedy.cu", "relations.cu", "table.cu", "noalloc.cu", "window.cu",
           "kv.cu", "kv_store.cu", "kv_rotate.cu", "kv_move.cu", "kv_tree.cu", "kv_rows.cu", "kv_tiles.cu", "kv_join.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
# host code is compiled without floating-point contraction (calibrate.h is exact fp32, op by op)
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "-Xcompiler", "-ffp-contract=off",
         "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build the library")


def _stale(out: str, deps) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    headers = [os.path.join(CSRC, "ps_internal.cuh"), os.path.join(CSRC, "calibrate.h"),
               os.path.join(CSRC, "greedy_grid.h"),
               os.path.join(ROOT, "include", "packserve.h")]
    kv_headers = [os.path.join(CSRC, "kv_internal.cuh"), os.path.join(CSRC, "kv_plan.h"),
                  os.path.join(CSRC, "kv_ring.h"), os.path.join(CSRC, "kv_elem.cuh"),
                  os.path.join(CSRC, "kv_turns.h"),
                  os.path.join(ROOT, "include", "packserve_kv.h"), headers[-1]]
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".cu", ".o"))
        if force or _stale(o, [s] + (kv_headers if src.startswith("kv") else headers)):
            cmd = [nvcc, *ARCH, *FLAGS, "-I", os.path.join(ROOT, "include"), "-c", s, "-o", o]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
            jobs.append(cmd)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
        return r.stdout + r.stderr

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        for out in ex.map(run, jobs):
            if verbose and out:
                sys.stderr.write(out)
    objs = [os.path.join(BUILD, s.replace(".cu", ".o")) for s in SOURCES]
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        run([nvcc, *ARCH, "-shared", "-o", tmp, *objs])
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
