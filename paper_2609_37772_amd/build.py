"""Build libuad.so (HIP, gfx950) in-tree.

    python -m paper_2609_37772_amd.build [--jobs N] [--debug]

Compiles every translation unit under csrc/ with hipcc for gfx950 and links
them into paper_2609_37772_amd/libuad.so, and the binding's argument checks
(csrc/marshal.c, host C) into _marshal.so, without which the binding makes them
in Python: it is left out where gcc or Python's headers are missing.  Always recompiles (no caching), so
a call after any source change is enough to refresh the library.
"""
from __future__ import annotations

import argparse
import concurrent.futures as cf
import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libuad.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"

COMMON = [
    f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-function",
    # code object v5: loadable by the HIP runtime that PyTorch bundles
    "-mcode-object-version=5",
    # keep hipcc from forming packed fp32 instructions (see the design notes)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(HERE, "..", "include"),
]


def _compile(src: str, extra) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [HIPCC, *COMMON, *extra, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    warn = "\n".join(ln for ln in r.stderr.splitlines() if "packed-fp32-ops" not in ln and ln.strip())
    if warn:
        sys.stderr.write(warn + "\n")
    return obj


def _compile_marshal() -> None:
    cmd = [os.environ.get("CC", "gcc"), "-O2", "-fPIC", "-shared", "-Wall", "-I", sysconfig.get_paths()["include"],
           os.path.join(CSRC, "marshal.c"), "-o", MARSHAL + ".tmp"]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
        why = (r.stderr or f"exit code {r.returncode}") if r.returncode else ""
    except OSError as e:
        why = str(e)
    if why:
        sys.stderr.write(f"left out: {MARSHAL}\n{' '.join(cmd)}\n{why}\n")
        if os.path.exists(MARSHAL):  # one of older sources may check something else
            os.remove(MARSHAL)
        return
    os.replace(MARSHAL + ".tmp", MARSHAL)


def build(jobs: int = 8, debug: bool = False, verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.cpp")))
    extra = ["-g"] if debug else []
    with cf.ThreadPoolExecutor(max_workers=max(1, jobs)) as ex:
        marshal = ex.submit(_compile_marshal)
        objs = list(ex.map(lambda s: _compile(s, extra), srcs))
        marshal.result()
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-mcode-object-version=5", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB} from {len(srcs)} sources")
    return LIB


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--jobs", type=int, default=8)
    ap.add_argument("--debug", action="store_true")
    a = ap.parse_args()
    build(a.jobs, a.debug)
