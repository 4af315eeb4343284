"""Build the C-ABI shared library in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libstrassen_b200.so")
SOURCES = ["plan.cpp", "add_kernels.cu", "add3_kernels.cu", "gemm_f64.cu", "fused_step.cu", "bfs_shares.cu", "bilinear.cu", "bilinear_plan.cpp", "probe.cu", "api.cu", "static_entry.cu", "tune.cu", "scale_kernels.cu",
           "rows8.cu", "route.cu", "w4_pack.cu", "w4_thin.cu", "w4_thin_bf16.cu", "w4_thin_f16.cu", "w4_thin_e4m3.cu", "w4_tiles.cu", "llm_api.cu",
           "kv_append.cu", "decode_attention.cu", "decode_bf16.cu", "decode_f16.cu", "decode_e4m3.cu", "prompt_attention.cu", "attention_api.cu"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every source for sm_100a and link libstrassen_b200.so next to this file."""
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(ROOT, "include", "strassen_b200.h"))
    nvcc = _nvcc()
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
        if force or _stale(o, [s] + headers):
            extra = ["-Xptxas", "-v"] if verbose else []
            jobs.append([nvcc] + NVCC_FLAGS + extra + ["-x", "cu", "-c", s, "-o", o])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed:\n%s\n%s" % (" ".join(cmd), r.stderr))
        return r.stderr

    with ThreadPoolExecutor(max_workers=4) as ex:
        for log in ex.map(run, jobs):
            if verbose and log:
                sys.stderr.write(log)
    objs = [os.path.join(OBJ, os.path.splitext(src)[0] + ".o") for src in SOURCES]
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + ".tmp%d" % os.getpid()
        run([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", tmp] + objs)
        os.replace(tmp, LIB)
    return LIB


def ensure_built() -> str:
    """The shared library, rebuilt first if it is absent or older than any source or header (used by the tests, the
    smoke check and the benchmark, so that what they run is what the sources say).  Where the library exists and no
    compiler does, it is used as it is."""
    try:
        return build()
    except OSError:          # no nvcc on this machine (a compile error is a RuntimeError and is not swallowed)
        if os.path.exists(LIB):
            return LIB
        raise


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
