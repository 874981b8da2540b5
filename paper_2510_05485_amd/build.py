"""Build the gfx950 shared library (libtensorbleu.so) and the Python module that calls it in-tree.

`python -m paper_2510_05485_amd.build` compiles every HIP translation unit under csrc/ for
gfx950 and links them into one C-ABI library next to this file, and csrc/tb_host.cpp,
csrc/loss/tb_loss_py.cpp and csrc/embed/tb_embed_py.cpp (host code, against PyTorch's headers) into the modules
_host, _loss_host and _embed_host.
hipcc cross-compiles without a GPU, so this runs anywhere the ROCm toolchain is installed.
"""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libtensorbleu.so")
HOST_SRC = os.path.join(CSRC, "tb_host.cpp")
HOST_LIB = os.path.join(PKG, "_host.so")
HOST_MODULES = [(HOST_SRC, HOST_LIB),
                (os.path.join(CSRC, "loss", "tb_loss_py.cpp"), os.path.join(PKG, "_loss_host.so")),
                (os.path.join(CSRC, "embed", "tb_embed_py.cpp"), os.path.join(PKG, "_embed_host.so"))]
FOLDERS = [CSRC, os.path.join(CSRC, "loss"), os.path.join(CSRC, "embed")]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
PRELOADED_WORDS = 14  # of a kernel's plain arguments
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the first 56 bytes of a kernel's plain arguments come in scalar registers
    "-mllvm", f"-amdgpu-kernarg-preload-count={PRELOADED_WORDS}", f"-DTB_PRELOADED_WORDS={PRELOADED_WORDS}",
    "-Wall", "-Wno-unused-function",
]


def sources():
    return sorted(f for folder in FOLDERS for f in glob.glob(os.path.join(folder, "*.hip")))


def needs_build() -> bool:
    built = [LIB] + [lib for _, lib in HOST_MODULES]
    if not all(os.path.exists(f) for f in built):
        return True
    t = min(os.path.getmtime(f) for f in built)
    deps = sources() + [src for src, _ in HOST_MODULES] + \
        [f for folder in (*FOLDERS, INCLUDE) for f in glob.glob(os.path.join(folder, "*.h"))]
    return any(os.path.getmtime(d) > t for d in deps)


def build(verbose: bool = True) -> str:
    tmp = LIB + f".tmp{os.getpid()}"
    extra = os.environ.get("TB_HIPCC_EXTRA", "").split()   # extra hipcc flags for experiments
    include = ["-I", INCLUDE, "-I", CSRC]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.check_call(cmd)

    # (the files side by side: 3 minutes instead of 8; tb_fused.hip and the three tb_loss_<type>.hip take nearly all)
    with tempfile.TemporaryDirectory() as objects, concurrent.futures.ThreadPoolExecutor(8) as pool:
        names = [os.path.join(objects, os.path.basename(f) + ".o") for f in sources()]
        list(pool.map(run, [[HIPCC, *FLAGS, *extra, *include, "-c", f, "-o", o] for f, o in zip(sources(), names)]))
        run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-rdc", "-o", tmp, *names])
    os.replace(tmp, LIB)
    for src, lib in HOST_MODULES:
        build_host(verbose, src, lib)
    return LIB


def build_host(verbose: bool = True, src: str = HOST_SRC, lib: str = HOST_LIB) -> str:
    """A module that marshals calls (_host, _loss_host, _embed_host): links against the library and PyTorch."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = [INCLUDE, *cpp_extension.include_paths(), os.path.join(rocm, "include"),
               sysconfig.get_paths()["include"]]
    tmp = lib + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[f"-isystem{d}" for d in include], "-o", tmp, src, "-L", PKG, "-ltensorbleu",
           "-L", torch_lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip",
           "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, lib)
    return lib


EXAMPLE_SRC = os.path.join(PKG, "example", "c_caller.c")
EXAMPLE_BIN = os.path.join(PKG, "c_caller")


def build_example(verbose: bool = True) -> str:
    """The plain-C caller of the ABI (gcc, HIP runtime only), linked against the library."""
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    cmd = [os.environ.get("CC", "gcc"), "-std=c99", "-O2", "-Wall", "-D__HIP_PLATFORM_AMD__",
           "-I", INCLUDE, "-I", os.path.join(rocm, "include"), EXAMPLE_SRC, "-L", PKG,
           "-ltensorbleu", "-L", os.path.join(rocm, "lib"), "-lamdhip64", "-lm",
           "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + os.path.join(rocm, "lib"), "-o", EXAMPLE_BIN]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return EXAMPLE_BIN


if __name__ == "__main__":
    build()
    build_example()
    print("built", LIB)
    sys.exit(0)
