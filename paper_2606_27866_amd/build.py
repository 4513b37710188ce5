"""Build libflexmoe.so (HIP, gfx950) and the _tensors module in-tree.

    python -m paper_2606_27866_amd.build

The library is one shared object holding every kernel and the C ABI of
include/flexmoe.h.  All device code is compiled with packed-fp32 arithmetic
disabled (-packed-fp32-ops); hipcc's host pass warns that it does not know
the feature, which is harmless.  _tensors.so (host code, g++ and torch's C++
headers) reads lists of tensors for the binding's optimizer and makes the outputs
of its operators on rows; without them the library is built all the same.
"""
from __future__ import annotations

import glob
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libflexmoe.so")
TENSORS = os.path.join(HERE, "_tensors.so")
TENSORS_SRC = os.path.join(CSRC, "tensor_table.cpp")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def headers():
    return sorted(glob.glob(os.path.join(CSRC, "*.h"))) + [os.path.join(ROOT, "include", "flexmoe.h")]


def compile_command(out: str, extra=()):
    return [HIPCC, "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-shared",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function",
            "-I", os.path.join(ROOT, "include"), "-o", out, *extra, *sources()]


def tensors_missing() -> str:
    """What _tensors.so needs and this machine does not have; empty if nothing."""
    torch = importlib.util.find_spec("torch")
    needs = {"g++": shutil.which("g++"), "torch": torch,
             "torch's C++ headers": torch and os.path.exists(os.path.join(os.path.dirname(torch.origin), "include", "torch", "csrc",
                                                                          "autograd", "python_variable.h")),
             "Python.h": os.path.exists(os.path.join(sysconfig.get_path("include"), "Python.h"))}
    return ", ".join(name for name, found in needs.items() if not found)


def tensors_command(out: str):
    import torch
    from torch.utils.cpp_extension import include_paths
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    inc = [*include_paths(), sysconfig.get_path("include")]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-o", out, TENSORS_SRC, *["-I" + p for p in inc], "-L" + lib,
            "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]


def build_tensors() -> str:
    tmp = TENSORS + ".tmp%d" % os.getpid()
    subprocess.run(tensors_command(tmp), check=True)
    os.replace(tmp, TENSORS)
    return TENSORS


def build(verbose: bool = False) -> str:
    build_library(verbose)
    missing = tensors_missing()
    if missing:
        sys.stderr.write("without _tensors.so, which the optimizer and the operators on rows need: no %s here\n" % missing)
    else:
        build_tensors()
    return LIB


def build_library(verbose: bool = False) -> str:
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = compile_command(tmp)
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "'-packed-fp32-ops' is not a recognized feature for this target"
    msgs = [ln for ln in (r.stdout + r.stderr).splitlines() if noise not in ln and ln.strip()]
    if r.returncode != 0:
        sys.stderr.write("\n".join(msgs) + "\n")
        raise RuntimeError("hipcc failed (%d)" % r.returncode)
    if msgs and verbose:
        print("\n".join(msgs))
    os.replace(tmp, LIB)
    return LIB


def is_stale() -> bool:
    def older(out, files):
        return not os.path.exists(out) or any(os.path.getmtime(f) > os.path.getmtime(out) for f in files)

    return older(LIB, sources() + headers()) or not tensors_missing() and older(TENSORS, [TENSORS_SRC])


if __name__ == "__main__":
    print(build(verbose=True))
