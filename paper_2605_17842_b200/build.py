"""Build libsnlp.so (the C-ABI CUDA library, nvcc for sm_100a) and _bind.so (the native half of the Python binding), in-tree."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
SRCS = [os.path.join(HERE, "csrc", f) for f in ("snlp.cu", "lm_head_static.cu", "kv4.cu")]
LIB = os.path.join(HERE, "libsnlp.so")
BIND_SRC = os.path.join(HERE, "csrc", "bind.cpp")
BIND = os.path.join(HERE, "_bind.so")


def _newest_source_mtime() -> float:
    newest = 0.0
    for root in (os.path.join(HERE, "csrc"), os.path.join(os.path.dirname(HERE), "include")):
        for f in os.listdir(root):
            if f != os.path.basename(BIND_SRC):
                newest = max(newest, os.path.getmtime(os.path.join(root, f)))
    return newest


def _run(cmd, what, verbose):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed building {what}")
    if verbose:
        print(r.stderr)


def build_bind(force: bool = False, verbose: bool = False) -> str:
    header = os.path.join(os.path.dirname(HERE), "include", "snlp.h")
    if not force and os.path.exists(BIND) and os.path.getmtime(BIND) >= max(os.path.getmtime(BIND_SRC), os.path.getmtime(header)):
        return BIND
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    includes = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(nvcc)), "include")]
    _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", *("-I" + i for i in includes), BIND_SRC, "-o", BIND,
          "-L" + HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu",
          "-lc10_cuda", "-lc10"], os.path.basename(BIND), verbose)
    return BIND


def build(force: bool = False, verbose: bool = False) -> str:
    if force or not os.path.exists(LIB) or os.path.getmtime(LIB) < _newest_source_mtime():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
               "-Xcompiler", "-fPIC,-O2", "-shared",
               "-o", LIB, *SRCS, "-lcudart", "-lcuda"]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        _run(cmd, os.path.basename(LIB), verbose)
    build_bind(force, verbose)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
