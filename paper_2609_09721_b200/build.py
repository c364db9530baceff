"""Builds the C-ABI CUDA library in-tree, paper_2609_09721_b200/libefq_b200.so (sm_100a only), and the CPython extensions
beside it that call it: efq_fastcall.so, which takes plain integers, and efq_tensorcall.so, which takes torch tensors."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libefq_b200.so")
FASTCALL_SRC = os.path.join(CSRC, "fastcall.c")
FASTCALL = os.path.join(_HERE, "efq_fastcall.so")
TENSORCALL_SRC = os.path.join(CSRC, "tensorcall.cpp")
TENSORCALL = os.path.join(_HERE, "efq_tensorcall.so")
BUILT_FOR = os.path.join(_HERE, "build", "efq_tensorcall.built_for")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
         "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def target() -> str:
    """What efq_tensorcall.so, which is compiled against torch's C++ headers, is good for."""
    import torch
    return f"torch {torch.__version__}, C++ ABI {int(torch._C._GLIBCXX_USE_CXX11_ABI)}, Python {sysconfig.get_config_var('EXT_SUFFIX')}"


def _built_for() -> str:
    if not os.path.exists(BUILT_FOR):
        return ""
    with open(BUILT_FOR) as f:
        return f.read()


def _stale() -> bool:
    built = (LIB, FASTCALL, TENSORCALL)
    if not all(os.path.exists(f) for f in built) or _built_for() != target():
        return True
    t = min(os.path.getmtime(f) for f in built)
    deps = sources() + [FASTCALL_SRC, TENSORCALL_SRC] + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def _start_tensorcall(out: str):
    import torch
    torch_dir = os.path.dirname(torch.__file__)
    return subprocess.Popen([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC",
                             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DEFQ_BUILT_FOR="{target()}"', "-I", sysconfig.get_paths()["include"],
                             "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(torch_dir, "include"), TENSORCALL_SRC, "-o", out,
                             "-L", os.path.join(torch_dir, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python"],
                            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds what is not up to date.  The library stands, and C programs have it, also where an extension beside it fails to build."""
    if not force and not _stale():
        return LIB
    os.makedirs(os.path.join(_HERE, "build"), exist_ok=True)
    tmp = {out: out + f".tmp{os.getpid()}" for out in (LIB, FASTCALL, TENSORCALL)}
    running = []

    def done(what, p):
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError(f"{p.args[0]} failed on {what}")

    try:
        running.append(_start_tensorcall(tmp[TENSORCALL]))
        objs, compiling = [], []
        for src in sources():
            objs.append(os.path.join(_HERE, "build", os.path.basename(src)[:-3] + ".o"))
            cmd = [NVCC, *FLAGS, "-c", src, "-o", objs[-1]] + (["-Xptxas", "-v"] if verbose else [])
            compiling.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
            running.append(compiling[-1][1])
        for src, p in compiling:
            done(src, p)
        subprocess.run([NVCC, "-shared", "-o", tmp[LIB], *objs, "-lcuda", "-cudart", "static"], check=True)
        os.replace(tmp[LIB], LIB)
        subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"],
                        "-I", os.path.join(ROOT, "include"), FASTCALL_SRC, "-o", tmp[FASTCALL]], check=True)
        os.replace(tmp[FASTCALL], FASTCALL)
        done(TENSORCALL_SRC, running[0])
        os.replace(tmp[TENSORCALL], TENSORCALL)
        with open(BUILT_FOR, "w") as f:
            f.write(target())
    finally:                # of a build that has failed: neither compilers that go on nor files that they were writing
        for p in running:
            if p.poll() is None:
                p.kill()
                p.communicate()
        for path in tmp.values():
            if os.path.exists(path):
                os.remove(path)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
