"""Compile the CUDA library in-tree: paper_2401_14021_b200/libralm.so (sm_100a only), and beside it the
tensor marshalling _native.so.

`--debug` builds libralm_debug.so beside it with -DRALM_DEBUG_BOUNDS: every index into a global
array that a scan kernel computes is checked against the array's extent (a violation is recorded
in the status word as RALM_ERR_INTERNAL; nothing traps); the generator's operators are in it as they are. Point RALM_LIBRARY at that file to run
the tests or the benchmark on it."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libralm.so")
DEBUG_LIB = os.path.join(HERE, "libralm_debug.so")
BINDING = os.path.join(HERE, "_native.so")      # tensor marshalling of the generator's operators
SOURCES = ["ralm_api.cu", "generate_api.cu", "os3.cpp"]
HEADERS = ["common.cuh", "scan.cuh", "aux_kernels.cuh", os.path.join("..", "..", "include", "ralm.h")]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    paths += [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    return max(os.path.getmtime(p) for p in paths if os.path.exists(p))


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    lib = DEBUG_LIB if debug else LIB
    if not debug:
        build_binding(force)
    if not force and os.path.exists(lib) and os.path.getmtime(lib) >= _newest_source_mtime():
        return lib
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = lib + ".tmp.%d" % os.getpid()
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "--threads", "0"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    if debug:
        cmd += ["-DRALM_DEBUG_BOUNDS"]
    cmd += [os.path.join(CSRC, f) for f in SOURCES] + ["-o", tmp, "-lcudart"]
    subprocess.run(cmd, check=True)
    os.replace(tmp, lib)
    return lib


def build_binding(force: bool = False) -> str:
    """Compile csrc/binding.cpp against the installed torch: paper_2401_14021_b200/_native.so."""
    source = os.path.join(CSRC, "binding.cpp")
    newest = max(os.path.getmtime(p) for p in (source, os.path.join(CSRC, "..", "..", "include", "ralm.h")))
    if not force and os.path.exists(BINDING) and os.path.getmtime(BINDING) >= newest:
        return BINDING
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    tmp = BINDING + ".tmp.%d" % os.getpid()
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC",
                    "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), source, "-o", tmp]
                   + ["-isystem" + i for i in include]
                   + ["-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"], check=True)
    os.replace(tmp, BINDING)
    return BINDING


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
