"""Build libpnerf.so (HIP, gfx950) in the package directory.

Every source is compiled with hipcc for gfx950 only; packed-FP32 instruction
selection is disabled (-packed-fp32-ops).  Sources are compiled in parallel and
linked into one shared library next to this file.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpnerf.so")
SOURCES = ["api.hip", "march.hip", "encode.hip", "mlp.hip", "composite.hip", "pose.hip",
           "layers_api.hip", "attention.hip", "attention_bwd.hip", "norm_rotate.hip", "linear.hip",
           "rotate_axes.hip", "attention_q8.hip", "quantize.hip", "layer_norm.hip", "clip.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-fhip-fp32-correctly-rounded-divide-sqrt", "-fno-gpu-rdc", "-ffp-contract=on",
         "-Wall", "-Wno-unused-function", "-Wno-unused-variable", "-Wno-unknown-pragmas",
         "-I", os.path.join(HERE, "..", "include")]

SOURCE_FLAGS = {
    # the encoding claims its next work item before it needs it: without this the
    # compiler broadcasts the atomic's result, and waits for it, at once
    "encode.hip": ["-mllvm", "-amdgpu-atomic-optimizer-strategy=None"],
}


def flags(src: str) -> list[str]:
    """The compiler flags of one source."""
    return FLAGS + SOURCE_FLAGS.get(src, [])


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, src.replace(".hip", ".o"))
    cmd = [HIPCC, *flags(src), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    # keep warnings visible but filter the host pass's note about the GPU-only feature
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if err.strip():
        print(err, file=sys.stderr)
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES), 8)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
