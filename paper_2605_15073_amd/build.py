"""Build libcgtp.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libcgtp.so")
SOURCES = ["plan.cpp", "tables.cpp", "order.cpp", "rows.cpp", "contract.hip", "contract_rows.hip", "kernels.hip", "onsite.hip", "receiver_mfma.hip",
           "receiver_values.hip", "folded.hip",
           "fourier_mfma.hip", "noalloc.hip", "group_rows.hip", "rows_product.hip", "rows_outer.hip", "rows_wide.hip", "layer_wide_bf16.hip", "layer_wide_f32.hip", "rows_few.hip", "rows_thin.hip", "layer_grad.hip", "rows_route.hip", "rows_mix.hip", "adamw.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# Per-source flags. The receivers' matrix-core results feed vector ALU products at once, those of
# the row products the conversion of a store: accumulating them in VGPRs (not AccVGPRs) saves a
# copy per result element and registers.
SOURCE_FLAGS = {src: ["-mllvm", "-amdgpu-mfma-vgpr-form"]
                for src in ("receiver_mfma.hip", "receiver_values.hip", "rows_product.hip",
                            "rows_outer.hip", "rows_wide.hip", "layer_wide_bf16.hip", "layer_wide_f32.hip",
                            "rows_thin.hip", "layer_grad.hip")}

# Packed fp32 VALU ops are disabled for all device code.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", INCLUDE, "-I", CSRC]


def build(verbose: bool = False) -> str:
    build_dir = os.path.join(HERE, "_build")
    os.makedirs(build_dir, exist_ok=True)
    objs = [os.path.join(build_dir, src + ".o") for src in SOURCES]

    def compile_one(src_obj):
        src, obj = src_obj
        cmd = [HIPCC, *FLAGS, *SOURCE_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    # one compiler process per source, at most as many as the host offers (16 at most)
    jobs = max(1, min(len(SOURCES), len(os.sched_getaffinity(0)), 16))
    with ThreadPoolExecutor(jobs) as pool:
        list(pool.map(compile_one, zip(SOURCES, objs)))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
    print(LIB)
