"""Build the HIP library in-tree for gfx950 (MI355X).

``python -m paper_2606_05933_amd.build`` (or ``__graft_entry__.build()``)
compiles ``csrc/*.hip`` and ``csrc/*.cpp`` into ``paper_2606_05933_amd/libssa.so``.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libssa.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

SOURCES = ["ssa_kernels.hip", "ssa_pool.hip", "ssa_layer.hip", "ssa_gemm.hip", "ssa_layer_forward.cpp", "ssa_scores.hip", "ssa_evict.hip", "ssa_evict_plan.cpp", "ssa_sparse.hip", "ssa_sparse_plan.cpp", "ssa_pages.hip", "ssa_probe.hip", "ssa_plan.cpp", "ssa_predictor.cpp", "ssa_scheduler.cpp"]
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
    # no packed-fp32 VALU forms anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # keep MFMA accumulators in VGPRs: the online-softmax rescale of the O tiles
    # is VALU work, and AGPR-homed accumulators cost two copies per key block
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-I", os.path.join(ROOT, "include"),
]


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"
    cmd = [HIPCC, *FLAGS, *[os.path.join(CSRC, s) for s in SOURCES], "-o", tmp]
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{err}")
    if verbose and err.strip():
        print(err, file=sys.stderr)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
