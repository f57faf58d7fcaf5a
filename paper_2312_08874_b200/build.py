"""Builds the CUDA library in-tree with nvcc for sm_100a (no torch extension machinery).

`python -m paper_2312_08874_b200.build` compiles every file of `csrc/` to an object under
`_build/` (in parallel) and links `libagent_attn.so` next to this file.  nvcc cross-compiles,
so no GPU is needed to build.
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys
from typing import List

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libagent_attn.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--use_fast_math", "-Xcompiler", "-fPIC", "-Xptxas", "-v",
]
# --use_fast_math serves the 16-bit kernels' divisions; the fp32 kernels keep IEEE division, logarithms and denormals, and exp2f
# where they call it (the term kernels' probabilities are explicit ex2.approx, as accurate on their range), so they go without.
PRECISE_FILES = {"attn_simt.cu", "pool.cu", "api.cu", "backward.cu", "bwd_terms.cu", "bwd_terms_umma.cu", "bwd_values_umma.cu", "rotate.cu", "gated.cu"} | {f"bwd_terms_d{d}.cu" for d in (32, 48, 64, 80, 96, 128)}


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _sources() -> List[str]:
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    paths.append(os.path.join(HERE, "..", "include", "agent_attn.h"))
    return max(os.path.getmtime(p) for p in paths)


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJ_DIR, src[:-3] + ".o")
    flags = [f for f in NVCC_FLAGS if not (src in PRECISE_FILES and f == "--use_fast_math")]
    cmd = [_nvcc()] + flags + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}")
    with open(obj + ".log", "w") as f:      # ptxas -v output: registers, spills, shared memory
        f.write(r.stdout)
    if verbose:
        print(r.stdout)
    return obj


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile and link the library if it is missing or older than its sources."""
    if not force and os.path.exists(LIB_PATH) and os.path.getmtime(LIB_PATH) >= _deps_mtime():
        return LIB_PATH
    os.makedirs(OBJ_DIR, exist_ok=True)
    srcs = _sources()
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
    cmd = [_nvcc(), "-shared", "-o", LIB_PATH] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}")
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
