"""Build libstepq.so in-tree with nvcc for sm_103a (one -gencode, TUs in parallel), and beside it
the compiled half of the Python binding, which needs the headers of the torch and the Python that it is used
with. The library needs neither."""
from __future__ import annotations

import concurrent.futures as cf
import hashlib
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

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


BIND_SOURCE = "bind.cpp"


def bind_so() -> str | None:
    """Where the binding for this Python and its torch is built (None: there is no torch). It is linked to the files of
    both, so each pair has its own."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    place = hashlib.sha256(os.path.realpath(spec.origin).encode()).hexdigest()[:8]
    name = "-".join(("torch", importlib.metadata.version("torch"), place, sysconfig.get_config_var("SOABI") or sys.implementation.cache_tag))
    return os.path.join(BUILD, name, "_stepq_bind.so")


def nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libstepq.so")


def _older(so: str, sources) -> bool:
    if not os.path.exists(so):
        return True
    t = os.path.getmtime(so)
    deps = [os.path.join(CSRC, f) for f in sources] + [os.path.join(INCLUDE, "stepq.h"), os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def _stale() -> bool:
    return _older(SO, SOURCES + HEADERS)


def build_bind(force: bool = False) -> str:
    so = bind_so()
    if so is None:
        raise RuntimeError("torch not found: the device calls take its tensors")
    if not force and not _older(so, [BIND_SOURCE]):
        return so
    os.makedirs(os.path.dirname(so), exist_ok=True)
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    tmp = so + f".{os.getpid()}.tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-I", INCLUDE, "-I", os.path.join(torch, "include"),
           "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include"), os.path.join(CSRC, BIND_SOURCE),
           "-o", tmp, "-L", os.path.join(torch, "lib"), "-ltorch_python", "-lc10", "-lc10_cuda",
           "-Wl,-rpath," + os.path.join(torch, "lib")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on {BIND_SOURCE}:\n{r.stderr}")
    os.replace(tmp, so)
    return so


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds what is older than its sources, the binding too if there is a torch; libstepq.so's path."""
    with cf.ThreadPoolExecutor(max_workers=1) as ex:
        bind = ex.submit(build_bind, force) if bind_so() else None
        so = build_library(force, verbose)
        if bind:
            bind.result()
    return so


def build_library(force: bool = False, verbose: bool = False) -> str:
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
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
