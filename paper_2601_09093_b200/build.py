"""Builds libstep.so (the C-ABI library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libstep.so")
STAMP = os.path.join(HERE, "_build", "libstep.stamp")
SOURCES = ["pool.cu", "attention.cu", "scorer.cu", "scorer_tc.cu", "prune.cu", "algorithm1.cu", "train.cu", "probe.cu",
           "tree.cu", "tree_tc.cu", "weights.cu", "evict.cu", "rotary.cu", "groups.cu", "groups_tc.cu"]
ARCH = ["-gencode", "arch=compute_100a,code=sm_100a"]
FLAGS = ARCH + ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-Xptxas", "-v"]
# Rotations keep subnormal numbers, which fast arithmetic flushes (same registers, same times); the others do without them.
PRECISE = ("rotary.cu",)


def _flags(source: str) -> list[str]:
    return FLAGS if source in PRECISE else FLAGS + ["--use_fast_math"]


def _nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: libstep.so cannot be built")
    return cand


def _digest() -> str:
    h = hashlib.sha256(" ".join(f for s in SOURCES for f in [s] + _flags(s)).encode())
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
    nvcc = _nvcc()

    def run(cmd):
        res = subprocess.run([nvcc] + cmd, capture_output=True, text=True)
        return res.returncode, res.stdout + res.stderr

    objects = [os.path.join(os.path.dirname(STAMP), s + ".o") for s in SOURCES]
    with ThreadPoolExecutor(os.cpu_count()) as pool:
        done = list(pool.map(run, [_flags(s) + ["-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objects)]))
    if not any(rc for rc, _ in done):
        done.append(run(ARCH + ["-shared", "-Xcompiler", "-fPIC"] + objects + ["-o", LIB]))
    log = "".join(text for _, text in done)
    with open(os.path.join(os.path.dirname(STAMP), "nvcc.log"), "w") as f:
        f.write(log)
    if any(rc for rc, _ in done):
        sys.stderr.write(log)
        raise RuntimeError("nvcc failed building libstep.so")
    if verbose:
        print(log)
    with open(STAMP, "w") as f:
        f.write(dig)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
