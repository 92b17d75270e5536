"""Compile the HIP library for gfx950 in-tree: ``python -m paper_2404_00509_amd.build``."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

from . import lds_reads

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
SOURCES = ["api.hip", "api_train.hip", "mask_params.hip", "crop_patch.hip", "normpix_loss.hip",
           "patch_embed.hip", "three_aug.hip", "jpeg_decode.hip", "layer_norm.hip", "dropout.hip",
           "class_loss.hip", "embed_grad.hip"]
OUT = os.path.join(_HERE, "libmae_hip.so")

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-shared", "-Wall", "-Wextra",
    # packed fp32 instructions are kept out of the generated code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    noise = "is not a recognized feature for this target"
    log = "\n".join(l for l in res.stdout.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + log)
    if verbose and log.strip():
        print(log, flush=True)


def compile_source(source: str, obj: str, verbose: bool = False) -> None:
    """One source to an object file.  With the matrix kernels' main loop in it, the assembly that the object is made
    of is checked first (lds_reads)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc] + [f for f in HIPCC_FLAGS if f != "-shared"] + ["-c", source, "-o", obj]
    with open(source) as f:
        checked = '#include "matmul.hpp"' in f.read()
    _run(cmd + ["-save-temps=obj"] if checked else cmd, verbose)
    if checked:
        stem = os.path.splitext(os.path.basename(source))[0]
        made = glob.glob(os.path.join(os.path.dirname(obj), stem + "-*gfx950*.s"))
        if len(made) != 1:
            raise RuntimeError(f"{stem}: the compiler left {len(made)} assembly files of the device code, expected one")
        with open(made[0]) as f:
            lds_reads.check(f.read(), os.path.basename(source))


def build_hip(verbose: bool = False) -> str:
    """The sources side by side, then one link (one after the other they take four times as long)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    jobs = max(1, min(8, os.cpu_count() or 1, int(os.environ.get("MAX_JOBS", "8") or 8)))
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(jobs) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        # (the longest first)
        order = sorted(range(len(SOURCES)), key=lambda i: -os.path.getsize(os.path.join(CSRC, SOURCES[i])))
        todo = [pool.submit(compile_source, os.path.join(CSRC, SOURCES[i]), objects[i], verbose) for i in order]
        for t in todo:
            t.result()
        _run([hipcc] + HIPCC_FLAGS + ["-o", OUT] + objects, verbose)
    return OUT


if __name__ == "__main__":
    print(build_hip(verbose=True))
    sys.exit(0)
