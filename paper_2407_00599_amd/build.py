"""Builds libparm_moe.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree.

    python -m paper_2407_00599_amd.build            # build if sources are newer than the library
    python -m paper_2407_00599_amd.build --force
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libparm_moe.so")
SOURCES = ["api.hip", "gate.hip", "permute.hip", "ffn.hip", "gate_bwd.hip", "schedule.hip", "ragged.hip",
           "ragged_few.hip", "ragged_f32.hip", "glu.hip", "mx4.hip", "mx4_few.hip", "mx4_tile.hip", "mx4_ffn.hip", "ckpt8.hip", "norm.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-fvisibility=default",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",   # no packed-fp32 VALU ops
    "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]
# The speed of the expert FFN's k loops depends on where in a 64-byte line of the instruction cache they start, and any edit in
# front of them moves them: the merged backward launch of 8 experts x 16384 x 4096 x 7168, same loops, 17.44 ms with a loop at
# the start of a line and 17.78 behind it; the call 21.96 / 22.19 / 21.90 ms (by chance aligned / moved / aligned by this).  The
# padding costs where short loops nest (slots of the gate 6.4 -> 6.6 us), so the other sources go without.
FILE_FLAGS = {f: ["-Xarch_device", "-falign-loops=64"] for f in ("ffn.hip", "ragged.hip", "glu.hip", "mx4_tile.hip")}


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "parm_moe.h"), __file__]
    return any(os.path.getmtime(d) > t for d in deps)


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = [HIPCC, *FLAGS, *FILE_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(force: bool = False, verbose: bool = True) -> str:
    if not force and not _stale():
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv)
