"""Builds libjorge.so (the HIP kernels and the C ABI) in-tree for gfx950."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libjorge.so")
SOURCES = [os.path.join(CSRC, f) for f in ("jorge.hip", "lm_api.hip", "lm_norm.hip", "lm_embed.hip", "lm_loss.hip",
                                           "lm_adamw.hip")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    # Keep the compiler from forming packed fp32 instructions.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", os.path.join(ROOT, "include"),
]


def _run(cmd: list[str], verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        sys.stderr.write(err + "\n")
        raise subprocess.CalledProcessError(res.returncode, cmd, res.stdout, res.stderr)
    if verbose and err.strip():
        sys.stderr.write(err + "\n")


def build_library(verbose: bool = False) -> str:
    """Compiles every source, side by side, and links libjorge.so; raises CalledProcessError on failure."""
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory() as objects, ThreadPoolExecutor(min(len(SOURCES), 8)) as pool:
        outs = [os.path.join(objects, os.path.basename(s) + ".o") for s in SOURCES]
        for done in [pool.submit(_run, [HIPCC, *FLAGS, "-c", s, "-o", o], verbose) for s, o in zip(SOURCES, outs)]:
            done.result()
        _run([HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared", *outs, "-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
