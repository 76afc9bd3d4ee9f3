"""Compiles the HIP sources in csrc/ into paper_2510_24211_amd/libscd.so for
gfx950 (hipcc cross-compiles without a GPU)."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libscd.so")
SOURCES = ["scd_api.hip", "lm_head.hip", "row.hip", "row_batched.hip", "row_short.hip", "commit.hip",
           "workload_gather.hip", "lm_head_quantized.hip",
           "embed.hip", "cross_entropy.hip", "lm_head_fp8.hip", "norm.hip", "clip.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
         # the method's fp32 roundings are part of its definition: no fused contraction
         "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # plain leading kernel arguments arrive in SGPRs at wavefront launch (the hot kernels put
         # what their first loads need there); kernels keep a fallback prologue that loads them
         "-mllvm", "-amdgpu-kernarg-preload-count=16",
         "-Wall", "-Wno-unused-function"]


def build(verbose=False, extra_flags=()):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, *FLAGS, *extra_flags, *[os.path.join(CSRC, s) for s in SOURCES], "-o", LIB]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines()
                    if "packed-fp32-ops" not in l)          # host pass does not know the feature
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    if verbose and out.strip():
        print(out)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, extra_flags=sys.argv[1:]))
