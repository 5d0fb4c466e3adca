"""Builds libstep.so (the C-ABI library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libstep.so")
STAMP = os.path.join(HERE, "_build", "libstep.stamp")
SOURCES = ["pool.cu", "attention.cu", "scorer.cu", "scorer_tc.cu", "prune.cu", "algorithm1.cu", "train.cu", "probe.cu",
           "tree.cu", "tree_tc.cu", "weights.cu", "evict.cu", "rotary.cu", "groups.cu", "groups_tc.cu"]
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "--use_fast_math", "-Xcompiler", "-fPIC", "-shared", "-Xptxas", "-v"]


def _nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: libstep.so cannot be built")
    return cand


def _digest() -> str:
    h = hashlib.sha256(" ".join(FLAGS).encode())
    files = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC))]
    files.append(os.path.join(os.path.dirname(HERE), "include", "step.h"))
    for f in files:
        with open(f, "rb") as fh:
            h.update(os.path.basename(f).encode() + b"\0" + fh.read())    # names, not paths: the tree may be moved
    return h.hexdigest()


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library if sources changed; returns the path of libstep.so."""
    dig = _digest()
    if not force and os.path.exists(LIB) and os.path.exists(STAMP) and open(STAMP).read() == dig:
        return LIB
    os.makedirs(os.path.dirname(STAMP), exist_ok=True)
    cmd = [_nvcc()] + FLAGS + [os.path.join(CSRC, s) for s in SOURCES] + ["-o", LIB]
    res = subprocess.run(cmd, capture_output=True, text=True)
    log = res.stdout + res.stderr
    with open(os.path.join(os.path.dirname(STAMP), "nvcc.log"), "w") as f:
        f.write(log)
    if res.returncode != 0:
        sys.stderr.write(log)
        raise RuntimeError("nvcc failed building libstep.so")
    if verbose:
        print(log)
    with open(STAMP, "w") as f:
        f.write(dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
