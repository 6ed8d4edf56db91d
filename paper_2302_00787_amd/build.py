"""Builds the HIP library in-tree: paper_2302_00787_amd/libfavorsharp.so (gfx950 only)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libfavorsharp.so")
OBJ = os.path.join(HERE, "_build")
COMMON = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
# Per-source extra flags.  Kernels that fit in 256 registers keep their MFMA results in ordinary vector registers
# (no accumulator-register copies before the exp2 / convert steps).  The files that use LDS float-maximum atomics from
# a few lanes switch the compiler's wave-level pre-reduction of atomics off (it would turn each into a lane loop).
SOURCES = {
    "favorsharp_api.hip": [],
    "kernels_generic.hip": [],
    "kernels_gen_walk.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_gen_small.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_gen_split.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_gen_rows.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_bf16.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-mllvm", "-amdgpu-atomic-optimizer-strategy=None"],
    "kernels_bf16_causal.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-mllvm", "-amdgpu-atomic-optimizer-strategy=None"],
    "kernels_bf16_bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-mllvm", "-amdgpu-atomic-optimizer-strategy=None"],
    "kernels_bf16_bwd_pc.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_bf16_wide.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_op.hip": [],
    "kernels_fit.hip": [],
    "state_api.hip": [],
    "kernels_rotary.hip": [],
    "kernels_state.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_state_rows.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
    "kernels_state_step.hip": [],
    "decay_api.hip": [],
    # (values that do not change in a loop are worked out there: kept for all turns they take registers that hold more waves otherwise)
    "kernels_decay.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1", "-mllvm", "-disable-machine-licm"],
    "kernels_decay_step.hip": [],
    "host_fit.cpp": [],
}


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the packed-fp32 target feature and says so; that line is noise
    err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
    if err.strip() and verbose:
        print(err, file=sys.stderr)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + err)


def build(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJ, exist_ok=True)
    objs = {src: os.path.join(OBJ, os.path.splitext(src)[0] + ".o") for src in SOURCES}
    with ThreadPoolExecutor(max_workers=4) as pool:       # (a compiler takes up to 2 GB)
        list(pool.map(lambda src: _run([hipcc, *COMMON, *SOURCES[src], "-x", "hip", "-c", os.path.join(CSRC, src), "-o", objs[src]], verbose),
                      SOURCES))
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs.values(), "-o", LIB], verbose)
    return LIB


if __name__ == "__main__":
    build()
