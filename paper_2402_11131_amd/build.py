"""Builds libss.so (the HIP kernels and their C ABI) for gfx950 with hipcc, and ss_bind.so (argument marshalling for Python)
with the host compiler."""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
INCLUDE = os.path.join(_ROOT, "include")
OBJ_DIR = os.path.join(_PKG, "_build")
LIB_PATH = os.path.join(_PKG, "libss.so")
BIND_PATH = os.path.join(_PKG, "ss_bind.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# Packed-fp32 VALU ops are switched off for all device code.
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument", "-I", INCLUDE, "-I", CSRC,
]


def _bind_command(out):
    """g++ line of ss_bind.so: torch's headers and libraries, no GPU code."""
    import torch
    base = os.path.dirname(torch.__file__)
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(),
            "-I", INCLUDE, "-isystem", os.path.join(base, "include"), "-I", sysconfig.get_paths()["include"],
            os.path.join(CSRC, "ss_bind.cpp"), "-L", os.path.join(base, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python", "-o", out]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _newer_than(path, deps):
    if not os.path.exists(path):
        return False
    t = os.path.getmtime(path)
    return all(os.path.getmtime(d) <= t for d in deps)


def build_lib(force: bool = True, verbose: bool = False, extra_flags=()) -> str:
    """Compile every csrc/*.hip and link libss.so, and ss_bind.so.  force=False skips
    what is newer than its sources and headers."""
    os.makedirs(OBJ_DIR, exist_ok=True)
    headers = glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    jobs = []
    objs = []
    for src in sources():
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-4] + ".o")
        objs.append(obj)
        if force or not _newer_than(obj, [src] + headers):
            jobs.append([HIPCC, *FLAGS, *extra_flags, "-c", src, "-o", obj])

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if r.returncode != 0:
            raise RuntimeError("%s failed:\n%s\n%s" % (os.path.basename(cmd[0]), " ".join(cmd), r.stdout))
        return r.stdout

    bind_tmp = BIND_PATH + ".tmp.%d" % os.getpid()
    bind = force or not _newer_than(BIND_PATH, [os.path.join(CSRC, "ss_bind.cpp"), os.path.join(INCLUDE, "ss.h")])
    if bind:
        jobs.insert(0, _bind_command(bind_tmp))
    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        list(ex.map(run, jobs))
    if bind:
        os.replace(bind_tmp, BIND_PATH)
    if len(jobs) > bind or not os.path.exists(LIB_PATH):
        tmp = LIB_PATH + ".tmp.%d" % os.getpid()
        run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs])
        os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    import sys
    print(build_lib(force="--force" in sys.argv, verbose=True))
