"""Build libflarepp.so (HIP, gfx950) in-tree with hipcc.

``python -m paper_2608_11519_amd.build`` compiles every source under
``csrc/`` into ``paper_2608_11519_amd/libflarepp.so``.
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libflarepp.so")
SOURCES = ["flarepp_kernels.hip", "flarepp_fused.hip", "flarepp_backward.hip",
           "flarepp_attn_bwd.hip", "flarepp_grad_gemm.hip", "flarepp_api.hip",
           "flarepp_linear.hip", "flarepp_linear_rows.hip", "flarepp_linear_bwd.hip",
           "flarepp_embedding.hip", "flarepp_adamw.hip", "flarepp_layers_api.hip"]
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (expected /opt/rocm/bin/hipcc)")


def command(out: str = LIB):
    return [
        hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
        # packed fp32 ops are kept out of the generated code on purpose
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        # MFMA accumulators in VGPRs: the softmax reads and rescales them with
        # VALU, and the AGPR form would copy them around every MFMA
        "-mllvm", "-amdgpu-mfma-vgpr-form=1",
        "-fvisibility=hidden", "-Wall", "-Wno-unused-result",
        "-parallel-jobs=8",  # of the sources below
        "-o", out,
    ] + [os.path.join(CSRC, s) for s in SOURCES]


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"
    cmd = command(tmp)
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed ({r.returncode}):\n{err}")
    if verbose and err.strip():
        print(err)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
