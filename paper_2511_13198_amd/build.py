"""Build the HIP library libpdyattn.so in-tree for gfx950 with hipcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libpdyattn.so")
SOURCES = [os.path.join(CSRC, f) for f in ("pdyattn.hip", "cross.hip", "rotary.hip")]
HEADERS = [os.path.join(CSRC, f) for f in ("common.hpp", "host.hpp", "plan.hpp", "fwd.hpp",
                                           "bwd.hpp", "cross.hpp", "cross_fwd.hpp", "cross_bwd.hpp",
                                           "rotary.hpp")] + [
    os.path.join(ROOT, "include", "pdyattn.h")]

ARCH = "gfx950"
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 VALU instructions anywhere in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False, extra_flags=None, out: str = LIB) -> str:
    """Every source compiled on its own, at the same time, then linked."""
    flags = [*FLAGS, *(extra_flags or []), "-I", os.path.join(ROOT, "include")]
    tmp = out + ".tmp"
    with tempfile.TemporaryDirectory() as work:
        objs, runs = [], []
        for src in SOURCES:
            objs.append(os.path.join(work, os.path.basename(src) + ".o"))
            runs.append(_start([hipcc(), *flags, "-c", "-o", objs[-1], src], verbose))
        for run in runs:
            _finish(run, verbose)
        _finish(_start([hipcc(), *flags, "-shared", "-o", tmp, *objs], verbose), verbose)
    os.replace(tmp, out)
    return out


def _start(cmd, verbose: bool) -> subprocess.Popen:
    if verbose:
        print(" ".join(cmd), flush=True)
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(run: subprocess.Popen, verbose: bool):
    text, _ = run.communicate()
    if run.returncode != 0:
        sys.stderr.write(text)
        raise RuntimeError(f"hipcc failed ({run.returncode})")
    if verbose and text.strip():
        sys.stderr.write(text)


if __name__ == "__main__":
    print(build(verbose=True))
