"""Build libcfp.so and libcfp_block.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcfp.so")
BLOCK_LIB = os.path.join(HERE, "libcfp_block.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    "-Wall",
    "-fvisibility=hidden",
    # keep the per-table switch cases of the register-resident kernel separate
    # (otherwise the cases are merged behind register copies)
    "-mllvm", "-simplifycfg-sink-common=false",
    # LDS atomics stay single instructions (no per-lane scalar loop)
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    # no packed fp32 instructions anywhere in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
    "-I", CSRC,
]


def sources(sub: str = ""):
    return sorted(glob.glob(os.path.join(CSRC, sub, "*.hip")))


def build(verbose: bool = False) -> str:
    """Compile every source to an object in parallel, then link: the search
    library from csrc/, the decoder-block operators from csrc/block/."""
    from concurrent.futures import ThreadPoolExecutor

    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    compile_flags = [f for f in FLAGS if f != "-shared"]

    def compile_one(src):
        obj = os.path.join(objdir, os.path.basename(src) + ".o")
        cmd = [HIPCC, *compile_flags, "-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)
        return obj

    libs = {LIB: sources(), BLOCK_LIB: sources("block")}
    srcs = [s for group in libs.values() for s in group]
    jobs = max(1, min(len(srcs), os.cpu_count() or 1, 16))
    with ThreadPoolExecutor(jobs) as ex:
        objs = dict(zip(srcs, ex.map(compile_one, srcs)))
    for lib, group in libs.items():
        tmp = lib + ".tmp"
        subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *(objs[s] for s in group), "-o", tmp])
        os.replace(tmp, lib)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)
