"""Builds libadacomp.so (HIP, gfx950 only) in-tree with hipcc."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libadacomp.so")
SOURCES = ["adacomp_api.hip", "adacomp_kernels.hip", "layers_api.hip", "layers_norm.hip", "layers_softmax.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off",                                     # no fused multiply-add, no reassociation
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",  # no packed-FP32 instructions
    # scalar arguments ahead of a kernel's structure are in registers when its workgroups start (k_pack, the unpack kernels)
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-Wall", "-Wextra",
]


def build(verbose: bool = False) -> str:
    """Compiles the sources side by side and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory(prefix="libadacomp_") as objects:
        def compile_one(source):
            out = os.path.join(objects, source + ".o")
            return out, subprocess.run([hipcc, *compile_flags, "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-c", "-o", out, os.path.join(CSRC, source)],
                                       capture_output=True, text=True)
        with concurrent.futures.ThreadPoolExecutor(max_workers=4) as pool:
            done = list(pool.map(compile_one, SOURCES))
        results = [res for _, res in done]
        if all(res.returncode == 0 for res in results):
            results.append(subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *[out for out, _ in done]],
                                          capture_output=True, text=True))
    for res in results:
        if verbose or res.returncode != 0:
            print(res.stdout)
            print(res.stderr)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed building libadacomp.so")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
