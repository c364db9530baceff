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
    if not force and not _stale():
        return LIB
    objs = []
    os.makedirs(os.path.join(_HERE, "build"), exist_ok=True)
    procs = []
    tensorcall_tmp = TENSORCALL + f".tmp{os.getpid()}"
    tensorcall = _start_tensorcall(tensorcall_tmp)
    for src in sources():
        obj = os.path.join(_HERE, "build", os.path.basename(src)[:-3] + ".o")
        cmd = [NVCC, *FLAGS, "-c", src, "-o", obj] + (["-Xptxas", "-v"] if verbose else [])
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.run([NVCC, "-shared", "-o", tmp, *objs, "-lcuda", "-cudart", "static"], check=True)
    os.replace(tmp, LIB)
    tmp = FASTCALL + f".tmp{os.getpid()}"
    subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"],
                    "-I", os.path.join(ROOT, "include"), FASTCALL_SRC, "-o", tmp], check=True)
    os.replace(tmp, FASTCALL)
    out, _ = tensorcall.communicate()
    if verbose or tensorcall.returncode != 0:
        sys.stderr.write(out)
    if tensorcall.returncode != 0:
        raise RuntimeError(f"g++ failed on {TENSORCALL_SRC}")
    os.replace(tensorcall_tmp, TENSORCALL)
    with open(BUILT_FOR, "w") as f:
        f.write(target())
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
