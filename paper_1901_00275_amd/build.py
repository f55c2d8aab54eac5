"""Builds libvlq.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libvlq.so")
SOURCES = ["api.hip", "coarse.hip", "coarse_bf16.hip", "coarse_half.hip", "train.hip", "search.hip", "scan_stream.hip", "scan_wide.hip", "encode.hip", "lists.hip",
           "softmax_loss.hip", "softmax_loss_narrow.hip", "softmax_loss_few.hip", "group_rows.hip", "clip_grads.hip"]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 instructions are not to be generated: some of their forms have given wrong results on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def _hipcc(*args: str) -> str:
    """What the compiler printed; RuntimeError if it failed"""
    res = subprocess.run(["hipcc", *FLAGS, *args], capture_output=True, text=True)
    out = "\n".join(l for l in (res.stdout + res.stderr).splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + out)
    return out


def build(verbose: bool = False) -> str:
    # a compiler per source, a few at a time, then one link
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        printed = list(pool.map(lambda s, o: _hipcc("-c", os.path.join(CSRC, s), "-o", o), SOURCES, objects))
        printed.append(_hipcc("-shared", "-o", LIB, *objects))
    out = "\n".join(p for p in printed if p.strip())
    if verbose and out:
        print(out)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
