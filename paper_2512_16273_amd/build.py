"""Builds the C-ABI library `libtslt.so` for gfx950 with hipcc (cross-compiles without a GPU), and, where there are a host
compiler and the headers of torch and Python, `_binding.so`, the fast path of the Python binding."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB_PATH = os.path.join(HERE, "libtslt.so")
BINDING_PATH = os.path.join(HERE, "_binding.so")
BINDING_SOURCE = os.path.join(HERE, "csrc", "binding.cpp")
SOURCES = [os.path.join(HERE, "csrc", n) for n in ("tslt.hip", "cache.hip", "attend_f32.hip", "attend_bf16.hip", "attend_f16.hip", "rotate.hip", "logprob.hip", "adapt.hip")]
HEADERS = [os.path.join(HERE, "csrc", n) for n in ("common.h", "bins.h", "handover.h", "pow_table.h", "truncate.h", "sample.h", "verify.h", "rowops.h", "rowsample.h", "exp64.h", "tree.h", "wire.h", "stats.h", "calib.h",
                                                   "error.h", "checks.h", "rows.h", "cache.h", "append.h", "attend.h", "attend_launch.h", "weigh.h", "evict.h", "rotate.h", "logprob.h", "adapt.h")] + \
          [os.path.join(ROOT, "include", "tslt.h")]


def hipcc_command(out: str = LIB_PATH, sources: list = SOURCES, kind: str = "-shared") -> list:
    """One command that makes `out` of `sources`; build_library compiles each source by one of its own, at the same time."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    return [hipcc, "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", kind,
            # packed-fp32 instructions are kept out of the generated code
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            # loop-invariant code motion after instruction selection: it carries fp64 constants through the tree
            # kernels' loops in vector registers, to the point of spilling (path of 64 trees 44 us with it, 39 without;
            # two trees, every node, 343 and 327)
            "-mllvm", "-disable-machine-licm",
            "-Wall", "-Wno-unused-function",
            "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc"),
            "-o", out] + list(sources)


def built_for() -> str:
    """What `_binding.so` depends on beside its source; the module carries it."""
    import torch
    return f"torch {torch.__version__}, Python {sys.version_info[0]}.{sys.version_info[1]}"


def binding_possible() -> bool:
    import torch
    headers = (os.path.join(os.path.dirname(torch.__file__), "include", "torch", "csrc", "autograd", "python_variable.h"),
               os.path.join(sysconfig.get_paths()["include"], "Python.h"))
    return shutil.which(os.environ.get("CXX", "g++")) is not None and all(os.path.exists(h) for h in headers)


def binding_command(out: str = BINDING_PATH) -> list:
    import torch
    base = os.path.dirname(torch.__file__)
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DTSLT_BUILT_FOR="{built_for()}"',
            "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(base, "include"),
            "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"), "-isystem", sysconfig.get_paths()["include"],
            "-o", out, BINDING_SOURCE, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]


def _run(commands: list, verbose: bool) -> None:
    """All of them at the same time; raises if one fails."""
    running = []
    for cmd in commands:
        if verbose:
            print(" ".join(cmd), flush=True)
        running.append((cmd, subprocess.Popen(cmd)))
    for cmd, process in running:
        process.wait()
    for cmd, process in running:
        if process.returncode != 0:
            raise subprocess.CalledProcessError(process.returncode, cmd)


def build_library(verbose: bool = True) -> str:
    bind = binding_possible()
    if not bind:
        print("no host compiler, or no headers of torch or Python: calls go through ctypes", flush=True)
        if os.path.exists(BINDING_PATH):
            os.remove(BINDING_PATH)                    # (of an earlier source, perhaps)
    with tempfile.TemporaryDirectory() as made:
        objects = [os.path.join(made, os.path.basename(s) + ".o") for s in SOURCES]
        _run([hipcc_command(o, [s], "-c") for s, o in zip(SOURCES, objects)] + ([binding_command()] if bind else []), verbose)
        hipcc = hipcc_command()[0]
        _run([[hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB_PATH] + objects], verbose)
    return LIB_PATH


def is_stale() -> bool:
    def older(out, sources):
        return not os.path.exists(out) or any(os.path.exists(s) and os.path.getmtime(s) > os.path.getmtime(out) for s in sources)
    if older(LIB_PATH, SOURCES + HEADERS):
        return True
    if not binding_possible():
        return False
    if older(BINDING_PATH, [BINDING_SOURCE, HEADERS[-1]]):
        return True
    with open(BINDING_PATH, "rb") as f:                # another torch or Python than it was built for
        return built_for().encode() + b"\0" not in f.read()


if __name__ == "__main__":
    build_library()
    print(LIB_PATH)
    sys.exit(0)
