"""Builds the C-ABI CUDA library in-tree: ``paper_2609_38166_b200/liblq.so`` for sm_100a.

``-fmad=false`` is part of the numerics contract: products are fused with additions only where the
kernels write fmaf(), which is what makes results reproducible bit for bit.
"""
from __future__ import annotations

import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblq.so")
# the same library with per-CTA time stamps compiled in (a development aid: bench.py --timeline reads them)
LIB_STAMPS = os.path.join(HERE, "liblq_stamps.so")
SOURCES = ["lq_api.cu", "lq_ops.cu", "lq_linear.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-fmad=false", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _headers(source: str, seen=None) -> set:
    """A source file and every file of this repository that it includes."""
    seen = set() if seen is None else seen
    if source not in seen:
        seen.add(source)
        with open(source) as f:
            for name in re.findall(r'^#include "([^"]+)"', f.read(), re.M):
                _headers(os.path.normpath(os.path.join(os.path.dirname(source), name)), seen)
    return seen


def _newest_source(source: str) -> float:
    return max(os.path.getmtime(p) for p in _headers(source))


def build(force: bool = False, verbose: bool = False, stamps: bool = False) -> str:
    """Compile if the library is missing or older than its sources; returns the library path.
    ``stamps``: the variant with the time stamps (-DLQ_TIMING -DLQ_STAMPS_ONLY) instead of the product."""
    LIB = LIB_STAMPS if stamps else globals()["LIB"]
    sources = [os.path.join(CSRC, f) for f in SOURCES]
    if not force and os.path.exists(LIB) and all(os.path.getmtime(LIB) >= _newest_source(s) for s in sources):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = ["-DLQ_TIMING", "-DLQ_STAMPS_ONLY"] if stamps else []
    objects, running = [], []
    for s in sources:                        # (an object that is newer than its sources is kept)
        o = s[:-3] + (".stamps.o" if stamps else ".o")
        objects.append(o)
        if force or not os.path.exists(o) or os.path.getmtime(o) < _newest_source(s):
            running.append((o, subprocess.Popen([nvcc, *NVCC_FLAGS, *extra, "-c", s, "-o", o + ".tmp"], stdout=subprocess.PIPE,
                                                stderr=subprocess.STDOUT, text=True)))
    said = [(o, p.communicate()[0], p.returncode) for o, p in running]
    for o, text, rc in said:
        if rc != 0:
            sys.stderr.write(text)
            raise RuntimeError("nvcc failed")
        if verbose:
            sys.stderr.write(text)
        os.replace(o + ".tmp", o)
    res = subprocess.run([nvcc, *NVCC_FLAGS[:2], "--shared", *objects, "-o", LIB + ".tmp"], capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed")
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    stamps_ = "--stamps" in sys.argv[1:]
    print(build(force=True, verbose=True, stamps=stamps_))
