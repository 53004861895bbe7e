"""Builds libdpb.so (HIP kernels for gfx950 + C ABI) in the package directory.

    python -m paper_2607_20652_amd.build

Each source compiles to its own object in parallel (under _build/ at the
repository root), then one link step writes the library.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdpb.so")
OBJ_DIR = os.path.join(os.path.dirname(HERE), "_build")
SOURCES = ["api.cpp", "api_around.cpp", "api_training.cpp", "tables.cpp", "adamw.hip", "attention.hip",
           "attention_bwd.hip", "cross_entropy.hip", "encode_general.hip", "embedding.hip", "codes.hip", "columns.hip",
           "columns_bwd.hip", "encode.hip", "extras.hip", "rms_norm.hip", "standardize.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]
# matrix-core results in ordinary VGPRs (no accumulator-register copies); not where they fill all 256
# accumulator registers and leave the ordinary ones to the operands
VGPR_FORM = ["-mllvm", "-amdgpu-mfma-vgpr-form"]
ACCUMULATORS = {"cross_entropy.hip"}
_NOISE = ("is not a recognized feature for this target", "argument unused during compilation")


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    msgs = "\n".join(l for l in (res.stdout + res.stderr).splitlines() if not any(n in l for n in _NOISE))
    return res.returncode, msgs


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    objs = [os.path.join(OBJ_DIR, os.path.splitext(s)[0] + ".o") for s in SOURCES]
    cmds = [[hipcc, *HIPCC_FLAGS, *([] if s in ACCUMULATORS else VGPR_FORM), "-c", os.path.join(CSRC, s), "-o", o]
            for s, o in zip(SOURCES, objs)]
    jobs = max(1, min(len(cmds), int(os.environ.get("MAX_JOBS", os.cpu_count() or 1))))
    with ThreadPoolExecutor(jobs) as ex:
        results = list(ex.map(_run, cmds))
    for cmd, (rc, msgs) in zip(cmds, results):
        if verbose:
            print(" ".join(cmd), flush=True)
        if rc != 0:
            raise RuntimeError(f"hipcc failed ({rc}) on {cmd[-3]}:\n{msgs}")
        if verbose and msgs.strip():
            print(msgs)
    tmp = LIB + ".tmp"
    rc, msgs = _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
    if rc != 0:
        raise RuntimeError(f"link failed ({rc}):\n{msgs}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
