"""Build the HIP library (C ABI of include/bpe.h, include/bpe_ops.h and include/bpe_head.h) for gfx950, in-tree."""
from __future__ import annotations

import glob
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbpe_hip.so")
SOURCES = [os.path.join(CSRC, "bpe.hip")]                       # the encoder
OPERATOR_SOURCES = [os.path.join(CSRC, "ops", "ops.hip")]       # the operators on token batches
HEAD_SOURCES = [os.path.join(CSRC, "head", name) for name in ("norm.hip", "project.hip", "adjust.hip")]      # a model's output end
INCLUDE = os.path.join(os.path.dirname(HERE), "include")


def headers():
    """Every header the library is compiled from: a change to any of them makes the built library stale."""
    return sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "ops", "*.h")) + glob.glob(os.path.join(CSRC, "head", "*.h")) + glob.glob(os.path.join(INCLUDE, "*.h")))

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-shared", "-fPIC",
    # packed fp32 instruction selection is switched off for every kernel of this library
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in SOURCES + OPERATOR_SOURCES + HEAD_SOURCES + headers())


def build(force: bool = True, extra_flags=()) -> str:
    """Compile csrc/*.hip into libbpe_hip.so with hipcc (cross-compiles without a GPU), the sources side by side."""
    if force or stale():
        hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
        with tempfile.TemporaryDirectory() as tmp:
            jobs, objects = [], []
            for source in SOURCES + OPERATOR_SOURCES + HEAD_SOURCES:
                objects.append(os.path.join(tmp, os.path.basename(source) + ".o"))
                flags = [f for f in HIPCC_FLAGS if f != "-shared"]
                jobs.append(subprocess.Popen([hipcc, *flags, *extra_flags, "-c", "-o", objects[-1], source]))
            failed = [j.args for j in jobs if j.wait() != 0]
            if failed:
                raise subprocess.CalledProcessError(1, failed[0])
            subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objects])
    return LIB


if __name__ == "__main__":
    print(build())
