"""Compile the HIP sources of this package into ``librsd.so`` and, with the table checks of every pass
switched on (``-DRSD_DEBUG``), ``librsd_debug.so`` (gfx950 only)."""
from __future__ import annotations

import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "librsd.so")
LIB_DEBUG = os.path.join(HERE, "librsd_debug.so")
ENGINE = os.path.join(HERE, "csrc", "rsd.hip")      # the engine (include/rsd.h)
OPERATORS = [os.path.join(HERE, "csrc", n) for n in ("ops.hip", "ops_kv.hip")]      # the operators (include/rsd_ops.h): 4-bit memory, the bf16 / fp32 cache
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc")]


def _start(cmd: list):
    return cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(jobs: list, verbose: bool) -> None:
    for cmd, proc in jobs:
        text, _ = proc.communicate()
        msgs = "\n".join(l for l in text.splitlines()
                         if "packed-fp32-ops" not in l)      # the host pass does not know the device feature
        if proc.returncode != 0:
            raise RuntimeError(f"hipcc failed: {' '.join(cmd[-4:])}\n" + msgs)
        if verbose and msgs.strip():
            print(msgs)


def build(verbose: bool = False) -> str:
    with tempfile.TemporaryDirectory() as tmp:
        eng, dbg = (os.path.join(tmp, n) for n in ("engine.o", "debug.o"))
        ops = [os.path.join(tmp, os.path.basename(src) + ".o") for src in OPERATORS]
        _finish([_start(["hipcc", *FLAGS, *extra, "-c", "-o", o, src])
                 for o, src, extra in ((eng, ENGINE, []), (dbg, ENGINE, ["-DRSD_DEBUG"]), *((o, src, []) for o, src in zip(ops, OPERATORS)))], verbose)
        _finish([_start(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", lib, o, *ops])
                 for lib, o in ((LIB, eng), (LIB_DEBUG, dbg))], verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
