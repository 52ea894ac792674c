"""Builds libss.so (the HIP kernels and their C ABI) for gfx950 with hipcc, and ss_bind.so (argument marshalling for Python)
with the host compiler."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
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


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("%s failed:\n%s\n%s" % (os.path.basename(cmd[0]), " ".join(cmd), r.stdout))


def build_lib(force: bool = True, verbose: bool = False, extra_flags=()) -> str:
    """Compile every csrc/*.hip and link libss.so: hipcc, nothing else.  force=False skips
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
    with ThreadPoolExecutor(max_workers=min(8, max(1, len(jobs)))) as ex:
        list(ex.map(lambda cmd: _run(cmd, verbose), jobs))
    if jobs or not os.path.exists(LIB_PATH):
        tmp = LIB_PATH + ".tmp.%d" % os.getpid()
        _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs], verbose)
        os.replace(tmp, LIB_PATH)
    return LIB_PATH


def build_bind(force: bool = True, verbose: bool = False) -> str:
    """Compile ss_bind.so: the host compiler, Python's and torch's headers.  force=False skips it if it is newer than its sources
    and was made for the torch and the Python that run (their ABIs are built in)."""
    import torch
    os.makedirs(OBJ_DIR, exist_ok=True)
    stamp_path = os.path.join(OBJ_DIR, "ss_bind.made_for")
    stamp = "\n".join((torch.__version__, sys.version, *_bind_command(BIND_PATH)))
    made_for = open(stamp_path).read() if os.path.exists(stamp_path) else None
    if force or made_for != stamp or not _newer_than(BIND_PATH, [os.path.join(CSRC, "ss_bind.cpp"), os.path.join(INCLUDE, "ss.h")]):
        tmp = BIND_PATH + ".tmp.%d" % os.getpid()
        _run(_bind_command(tmp), verbose)
        os.replace(tmp, BIND_PATH)
        with open(stamp_path, "w") as f:
            f.write(stamp)
    return BIND_PATH


def build_all(force: bool = True, verbose: bool = False) -> str:
    """Both, side by side; libss.so is there also where ss_bind.so cannot be built, which raises.  Returns libss.so's path."""
    with ThreadPoolExecutor(max_workers=1) as ex:
        bind = ex.submit(build_bind, force, verbose)
        path = build_lib(force, verbose)
        bind.result()
    return path


if __name__ == "__main__":
    # --lib: libss.so alone, for programs that use the C interface
    build = build_lib if "--lib" in sys.argv else build_all
    print(build(force="--force" in sys.argv, verbose=True))
