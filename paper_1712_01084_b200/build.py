"""Compile the CUDA sources under csrc/ into libpp_b200.so (sm_100a only), and csrc/torch/ into _pp_torch.so, the entry of the
decoder operators for PyTorch tensors."""
from __future__ import annotations

import glob
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpp_b200.so")
TORCH_SRC = os.path.join(CSRC, "torch", "pp_torch.cpp")
TORCH_LIB = os.path.join(HERE, "_pp_torch.so")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def needs_build_torch() -> bool:
    """Whether the extension module is missing, older than its sources or made for another PyTorch: its C++ interface is
    that of one version, whose name the module holds."""
    import torch
    if not os.path.exists(TORCH_LIB):
        return True
    if os.path.getmtime(TORCH_LIB) < max(os.path.getmtime(TORCH_SRC), os.path.getmtime(os.path.join(ROOT, "include", "pp.h"))):
        return True
    with open(TORCH_LIB, "rb") as f:
        return f"made for torch {torch.__version__}\0".encode() not in f.read()


def build_torch(force: bool = False) -> str:
    """The extension module: plain C++ against the headers of the installed PyTorch."""
    if not force and not needs_build_torch():
        return TORCH_LIB
    import sysconfig
    import torch
    base = torch.__path__[0]
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(ROOT, "include"), os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    lib = os.path.join(base, "lib")
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                           f'-DPP_TORCH_VERSION="made for torch {torch.__version__}"'] +
                          [x for d in include for x in ("-isystem" if d.startswith(base) else "-I", d)] +
                          ["-o", TORCH_LIB, TORCH_SRC, "-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda",
                           "-lc10"])
    return TORCH_LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """The library alone, which needs nvcc and no PyTorch."""
    if not force and not needs_build():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "--threads", "0", "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB] + sources() + ["-lcuda"]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_torch(force="--force" in sys.argv))
