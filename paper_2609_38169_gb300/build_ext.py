"""Build libstepq.so in-tree with nvcc for sm_103a (one -gencode, TUs in parallel)."""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
SO = os.path.join(BUILD, "libstepq.so")
INCLUDE = os.path.join(ROOT, "include")
SOURCES = ["plan.cpp", "api.cpp", "errors.cu", "stepq_kernels.cu", "heads.cu", "rows.cu", "baselines.cu", "intb.cu", "temporal.cu", "fp32.cu", "prefill.cu",
           "calib.cu", "calibrate.cu", "linattn.cpp", "linattn_decode.cu", "linattn_prefill.cu",
           "linattn_plan.cu", "linattn_chunks.cu", "linattn_terms.cu", "groupnorm.cu",
           "kv.cpp", "kv_rows.cu", "kv_attend_bf16.cu", "kv_attend_f16.cu", "kv_attend_int8.cu", "kv_attend_int4.cu"]
HEADERS = ["internal.h", "device.cuh", "async.cuh", "pipeline.cuh", "tile.cuh", "tcgen05.cuh", "linattn.cuh", "linattn_prefill.cuh",
           "kv.cuh", "kv_attend.cuh", "kv_launch.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libstepq.so")


def _stale() -> bool:
    if not os.path.exists(SO):
        return True
    t = os.path.getmtime(SO)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(INCLUDE, "stepq.h"),
                                                               os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return SO
    os.makedirs(BUILD, exist_ok=True)
    nv = nvcc()
    common = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-cudart", "shared",
              "-I", INCLUDE, "-I", CSRC] + ARCH
    if verbose:
        common += ["-Xptxas", "-v"]

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, src.rsplit(".", 1)[0] + ".o")
        cmd = [nv, "-c", os.path.join(CSRC, src), "-o", obj] + common
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = SO + f".{os.getpid()}.tmp"
    # the shared CUDA runtime: the library then sees the device and context torch uses
    cudalib = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nv))), "lib64")
    cmd = [nv, "-shared", "-cudart", "shared", "-Xlinker", f"-rpath={cudalib}", "-o", tmp] + objs + ARCH
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, SO)
    return SO


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
