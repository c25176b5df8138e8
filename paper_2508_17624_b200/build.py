"""Compile the CUDA sources into paper_2508_17624_b200/libexpertweave.so for sm_100a (in-tree)."""
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libexpertweave.so")
SOURCES = ["ew_vmm.cpp", "ew_pool.cu", "ew_route.cu", "ew_router.cu", "ew_gemm.cu", "ew_ablate.cu", "ew_ops.cu", "ew_grouped.cu", "ew_quant.cu",
           "ew_swiglu.cu", "ew_blocks.cu", "ew_norm.cu", "ew_scaled.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "expertweave.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    compile_ = [_nvcc(), "-c", "-Xcompiler", "-fPIC", *arch, "-lineinfo", "-O3", "-std=c++17", "-cudart", "static"]
    if verbose:
        compile_ += ["-Xptxas", "-v"]
    with tempfile.TemporaryDirectory() as objects:
        def one(source):
            target = os.path.join(objects, source + ".o")
            subprocess.run([*compile_, "-o", target, os.path.join(CSRC, source)], check=True)
            return target

        with ThreadPoolExecutor(max_workers=os.cpu_count() or 1) as pool:    # a file each
            targets = list(pool.map(one, SOURCES))
        subprocess.run([_nvcc(), "-shared", "-Xcompiler", "-fPIC", *arch, "-cudart", "static", "-o", LIB + ".tmp", *targets], check=True)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
