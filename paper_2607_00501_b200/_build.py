"""Build libqmm.so in-tree with nvcc for sm_100a (no other target is built), and beside it the CPython extensions
that marshal the arguments of its hot-path calls.  They are separate: the library serves every other call without an extension."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libqmm.so")
EXT = os.path.join(HERE, "_qmm_py" + sysconfig.get_config_var("EXT_SUFFIX"))      # (another CPython does not load it)
LAYER_EXT = os.path.join(HERE, "_qmm_layer_py" + sysconfig.get_config_var("EXT_SUFFIX"))
SOURCES = ("qmm_api.cu", "qmm_pack.cu", "qmm_gemv.cu", "qmm_gemm.cu", "qmm_gemm_small.cu", "qmm_moe.cu", "qmm_chain.cu",
           "qmm_mx_api.cu", "qmm_mx_quant.cu", "qmm_mx_gemm.cu", "qmm_expert.cu", "qmm_layer_api.cu", "qmm_router.cu", "qmm_norm.cu", "qmm_lora_f16.cu",
           "qmm_lora_bf16.cu", "qmm_lora_grad_f16.cu", "qmm_lora_grad_f16_rows8.cu", "qmm_lora_grad_bf16.cu", "qmm_lora_grad_bf16_rows8.cu")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
              "-Xcompiler", "-fPIC", "-DQMM_BUILD"]


def _nvcc() -> str:
    for p in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc"):
        if p and os.path.exists(p):
            return p
    return "nvcc"


def _stale(target: str, sources) -> bool:
    """Whether the target is missing or older than the C header or one of these files of csrc/."""
    files = [os.path.join(CSRC, f) for f in sources] + [os.path.join(os.path.dirname(HERE), "include", "qmm.h")]
    return not os.path.exists(target) or os.path.getmtime(target) < max(os.path.getmtime(f) for f in files)


def build(force: bool = False, verbose: bool = False) -> str:
    """libqmm.so and the extensions, beside this file."""
    build_library(force, verbose)
    build_extension(force)
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ and link libqmm.so."""
    if not force and not _stale(LIB, [f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))]):
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    hdr_time = max(os.path.getmtime(os.path.join(CSRC, f)) for f in os.listdir(CSRC) if f.endswith(".cuh"))
    hdr_time = max(hdr_time, os.path.getmtime(os.path.join(os.path.dirname(HERE), "include", "qmm.h")))

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, src.replace(".cu", ".o"))
        s = os.path.join(CSRC, src)
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(s), hdr_time):
            extra = os.environ.get("QMM_NVCC_EXTRA", "").split()     # e.g. -DQMM_GEMV_UNROLL=3 for tuning sweeps
            cmd = [nvcc] + NVCC_FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", obj]
            r = subprocess.run(cmd, capture_output=True, text=True)
            if verbose or r.returncode:
                sys.stderr.write(r.stdout + r.stderr)
            if r.returncode:
                raise RuntimeError("nvcc failed on %s" % src)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [nvcc, "-shared", "-o", tmp] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


def build_extension(force: bool = False) -> str:
    """Compile csrc/qmm_py.c and csrc/qmm_layer_py.c; the extensions find libqmm.so beside themselves."""
    for target, source in ((EXT, "qmm_py.c"), (LAYER_EXT, "qmm_layer_py.c")):
        if not force and not _stale(target, [source, "qmm_py.h"]):
            continue
        tmp = target + ".tmp.%d" % os.getpid()
        cmd = ["gcc", "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], os.path.join(CSRC, source), "-o", tmp,
               "-L", HERE, "-l:libqmm.so", "-Wl,-rpath,$ORIGIN"]
        subprocess.run(cmd, check=True)
        os.replace(tmp, target)
    return EXT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
