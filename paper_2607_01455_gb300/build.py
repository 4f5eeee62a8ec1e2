"""Compile libember.so (the CUDA library behind include/ember.h) for sm_103a.

Each .cu file compiles to an object in parallel, then nvcc links the shared
library in place under paper_2607_01455_gb300/_lib/.  nvcc cross-compiles, so
this runs on a machine without a GPU too.  Beside it: the operators' binding
to torch tensors, host code compiled against the headers of the torch at hand.
"""
import concurrent.futures
import os
import shutil
import subprocess
import sysconfig
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB_DIR = os.path.join(PKG, "_lib")
LIB = os.path.join(LIB_DIR, "libember.so")

NVCC = os.environ.get("NVCC", "nvcc")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-O2",
         "-I", INCLUDE, "-I", CSRC, "--expt-relaxed-constexpr"]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    return sources() + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))] + \
        [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE) if f.endswith(".h")]


def _compile(src, extra, objdir):
    obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
    subprocess.run([NVCC, *ARCH, *FLAGS, *extra, "-c", src, "-o", obj], check=True)
    return obj


def build_library(force: bool = False, verbose_ptxas: bool = False) -> str:
    """Build libember.so unless it is newer than every source and header."""
    if (not force and not verbose_ptxas and os.path.exists(LIB)
            and os.path.getmtime(LIB) >= max(os.path.getmtime(p) for p in _deps())):
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    os.makedirs(LIB_DIR, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose_ptxas else []
    # objects of concurrent builds (parallel test workers) never collide
    with tempfile.TemporaryDirectory(dir=BUILD) as objdir:
        with concurrent.futures.ThreadPoolExecutor(max_workers=len(sources())) as ex:
            objs = list(ex.map(lambda s: _compile(s, extra, objdir), sources()))
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.run([NVCC, *ARCH, "-shared", "-o", tmp, *objs], check=True)
        os.replace(tmp, LIB)
    return LIB


def binding_path() -> str:
    """Where the operators' binding for this interpreter and the torch at hand
    belongs: it fits the libraries of the torch that it was built against alone."""
    import torch
    return os.path.join(LIB_DIR, f"_ops_binding.{sysconfig.get_config_var('SOABI')}.torch-{torch.__version__}.so")


def build_binding(force: bool = False) -> str:
    """Build the operators' binding for the torch at hand unless it is there and newer than its source."""
    import torch
    binding = binding_path()
    src = os.path.join(CSRC, "ops_binding.cpp")
    if (not force and os.path.exists(binding)
            and os.path.getmtime(binding) >= max(os.path.getmtime(p) for p in (src, os.path.join(INCLUDE, "ember.h")))):
        return binding
    os.makedirs(LIB_DIR, exist_ok=True)
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(NVCC) or "/usr/local/cuda/bin/nvcc")))
    dirs = [INCLUDE, sysconfig.get_paths()["include"], os.path.join(home, "include"),
            os.path.join(home, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    libs = os.path.join(home, "lib")
    tmp = binding + f".tmp{os.getpid()}"
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    *(a for d in dirs for a in ("-I", d)), src, "-o", tmp, "-L", libs, "-lc10", "-lc10_cuda",
                    "-ltorch_cpu", "-ltorch", "-ltorch_python", f"-Wl,-rpath,{libs}"], check=True)
    os.replace(tmp, binding)
    return binding


if __name__ == "__main__":
    import sys
    print(build_library(force=True, verbose_ptxas="-v" in sys.argv))
    print(build_binding(force=True))
