"""Builds the HIP library in-tree for gfx950: python -m paper_2510_00206_amd.build"""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblorafusion_hip.so")
SOURCES = ["lf_api.hip", "lf_down.hip", "lf_gemm.hip", "lf_gemm_ring.hip", "lf_stream.hip", "lf_da.hip", "lf_ds.hip", "lf_unfused.hip", "lf_ceiling.hip",
           "lf_serve_api.hip", "lf_requests.hip", "lf_rope.hip", "lf_cache.hip", "lf_attn.hip",
           "lf_append.hip", "lf_weights.hip", "lf_layer4.hip"]
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]


def build_library(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    srcs = [os.path.join(CSRC, s) for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]
    cmd = [hipcc] + FLAGS + srcs + ["-o", LIB]
    if verbose:
        print(" ".join(cmd))
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops"
    err = "\n".join(ln for ln in res.stderr.splitlines() if noise not in ln)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)
    if verbose and err.strip():
        print(err)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose="-q" not in sys.argv))
