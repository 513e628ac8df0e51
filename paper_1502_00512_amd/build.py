"""Compiles the HIP sources into paper_1502_00512_amd/librnnlm_hip.so for gfx950."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librnnlm_hip.so")
SOURCES = [os.path.join(CSRC, "rnnlm.hip"), os.path.join(CSRC, "logit_ops.hip"),
           os.path.join(CSRC, "adapt_ops.hip")]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function"]


def _hipcc(args: list[str], verbose: bool) -> None:
    r = subprocess.run(["hipcc"] + args, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + msgs)
    if verbose and msgs.strip():
        print(msgs)


def build(verbose: bool = False) -> str:
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor() as pool:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        list(pool.map(lambda so: _hipcc(FLAGS + ["-c", so[0], "-o", so[1]], verbose), zip(SOURCES, objects)))
        _hipcc(["--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB] + objects, verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
