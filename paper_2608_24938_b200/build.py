"""Builds libexfold.so (sm_100a only) in-tree with nvcc.

    python -m paper_2608_24938_b200.build [--force] [--verbose]

Each .cu under csrc/ is compiled to an object file (in parallel) and linked into
paper_2608_24938_b200/libexfold.so. nvcc cross-compiles without a GPU.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "build")
LIB = os.path.join(HERE, "libexfold.so")
SOURCES = ["api.cu", "route_prefill.cu", "route_decode.cu", "combine_router.cu", "router_gemm.cu", "ffn_f32.cu", "calibrate.cu", "gemm_prefill.cu",
           "gemm_pair.cu", "gemm_mixed.cu", "ffn_decode.cu", "decode_small.cu", "no_alloc.cu",
           "route_general.cu", "route_given.cu", "linear.cu", "linear_small.cu", "linear_tile.cu", "linear_pair.cu"]
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]


def _newest_source_mtime() -> float:
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    files.append(os.path.join(HERE, "..", "include", "exfold.h"))
    return max(os.path.getmtime(f) for f in files)


def build(force: bool = False, verbose: bool = False, extra_flags=(), lib_path: str = LIB, obj_dir: str = OBJ) -> str:
    """extra_flags / lib_path / obj_dir let a debug variant (e.g. -DEXFOLD_TRACE) be built beside the product."""
    sources = list(SOURCES)
    LIB, OBJ = lib_path, obj_dir  # noqa: N806
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    flags = list(FLAGS) + list(extra_flags)
    if verbose:
        flags = flags + ["-Xptxas", "-v"]

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ, src.replace(".cu", ".o"))
        cmd = [NVCC, *flags, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(max(1, min(len(sources), os.cpu_count() or 1))) as ex:
        objs = list(ex.map(compile_one, sources))
    tmp = LIB + f".{os.getpid()}.tmp"
    rdc = ["-rdc=true"] if "-rdc=true" in flags else []
    r = subprocess.run([NVCC, "-shared", "-o", tmp, *objs, "-gencode", "arch=compute_100a,code=sm_100a", *rdc],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
