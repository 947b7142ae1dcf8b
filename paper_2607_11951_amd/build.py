"""Builds libgrid.so in-tree (host C++ with g++, kernels with hipcc for gfx950) and, where torch is installed, the Python
module _step on it."""

import importlib.util
import os
import subprocess
import sysconfig
from pathlib import Path

PKG = Path(__file__).resolve().parent
CSRC = PKG / "csrc"
OUT = PKG / "libgrid.so"
MODULE = PKG / "_step.so"
BUILD = PKG / "_build"
HOST_SOURCES = ["grammar.cpp", "lexer.cpp", "parser.cpp", "artifacts.cpp", "advance.cpp", "complete.cpp", "capi.cpp"]
HIP_SOURCES = ["kernels.hip", "paged.hip", "append.hip", "attend.hip", "attend_tree.hip", "verify.hip", "sample.hip",
               "tree.hip", "pages.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
HIP_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
HOST_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-pthread", "-Wall", "-Wextra", "-Wno-unused-parameter"]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(str(c) for c in cmd), flush=True)
    subprocess.run([str(c) for c in cmd], check=True)


def build(verbose=False, jobs=8):
    BUILD.mkdir(exist_ok=True)
    objs = []
    procs = []
    # torch's headers and libraries, found without importing it
    spec = importlib.util.find_spec("torch")
    if spec is not None:
        torch = Path(spec.origin).parent
        step = BUILD / "step_module.cpp.o"
        cmd = ["g++", *HOST_FLAGS, "-D__HIP_PLATFORM_AMD__=1", "-isystem", torch / "include",
               "-isystem", sysconfig.get_paths()["include"], "-isystem", "/opt/rocm/include", "-c",
               CSRC / "step_module.cpp", "-o", step]
        if verbose:
            print(" ".join(str(c) for c in cmd), flush=True)
        procs.append(subprocess.Popen([str(c) for c in cmd]))
    for src in HOST_SOURCES:
        obj = BUILD / (src + ".o")
        cmd = ["g++", *HOST_FLAGS, "-c", CSRC / src, "-o", obj]
        if verbose:
            print(" ".join(str(c) for c in cmd), flush=True)
        procs.append(subprocess.Popen([str(c) for c in cmd]))
        objs.append(obj)
    for src in HIP_SOURCES:
        obj = BUILD / (src + ".o")
        cmd = [HIPCC, *HIP_FLAGS, "-c", CSRC / src, "-o", obj]
        if verbose:
            print(" ".join(str(c) for c in cmd), flush=True)
        procs.append(subprocess.Popen([str(c) for c in cmd]))
        objs.append(obj)
    bad = [p.args for p in procs if p.wait() != 0]
    if bad:
        raise RuntimeError(f"compile failed: {bad}")
    tmp = str(OUT) + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-pthread", "-o", tmp, *objs], verbose)
    os.replace(tmp, OUT)
    if spec is not None:
        tmp = str(MODULE) + ".tmp"
        _run(["g++", "-shared", "-fPIC", "-o", tmp, step, f"-L{PKG}", "-l:libgrid.so", f"-L{torch / 'lib'}",
              "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip", "-Wl,-rpath,$ORIGIN"], verbose)
        os.replace(tmp, MODULE)
    return OUT


if __name__ == "__main__":
    build(verbose=True)
