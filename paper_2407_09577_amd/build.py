"""Build ``libflashnorm.so`` (gfx950) in-tree with hipcc, and the Python entry points on top of it.

Every ``csrc/*.hip`` file is compiled for gfx950 only, in parallel, then linked
into one shared library next to this file.  Packed-fp32 VALU instructions are
disabled for all device code (the kernels use scalar fp32 arithmetic).
``csrc/binding.cpp`` (host code, against the installed torch, with the C++ compiler of
``$CXX``) becomes the extension module ``_binding`` beside it; the library does not need it.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libflashnorm.so")
BINDING_PATH = os.path.join(HERE, "_binding.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")
ARCH = "gfx950"

CFLAGS = [
    "-O3", f"--offload-arch={ARCH}", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = [HIPCC, *CFLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    return obj


def _compile_binding() -> str:
    import torch
    from torch.utils import cpp_extension
    src, obj = os.path.join(CSRC, "binding.cpp"), os.path.join(BUILD_DIR, "binding.cpp.o")
    paths = [*cpp_extension.include_paths("cuda"), sysconfig.get_paths()["include"], INCLUDE]
    cmd = [CXX, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *(f"-isystem{p}" for p in paths), "-c", src,
           "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{CXX} failed for {src}:\n{r.stderr}")
    return obj


def _link_binding(obj: str) -> None:
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = BINDING_PATH + f".tmp{os.getpid()}"
    cmd = [CXX, "-shared", obj, f"-L{HERE}", "-l:libflashnorm.so", f"-L{libs}", "-ltorch_python", "-ltorch_cpu", "-ltorch_hip",
           "-lc10", "-lc10_hip", "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{libs}", "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, BINDING_PATH)


def _link_library(objs) -> None:
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    if os.path.exists(BINDING_PATH):
        os.remove(BINDING_PATH)  # made for the library before this one
    os.replace(tmp, LIB_PATH)


def build_binding() -> None:
    """Compile and link the binding alone, against the library that is there."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    _link_binding(_compile_binding())


def build(verbose: bool = True, binding: bool = True) -> str:
    """Compile every source and link the library, then the binding; always rebuilds.  The library needs hipcc alone:
    where the binding cannot be built the library stands before the error is raised, and where there is no torch (or
    binding is False) it is all that is built."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    binding = binding and importlib.util.find_spec("torch") is not None
    workers = min(len(srcs) + 1, max(1, (os.cpu_count() or 4)), 8)
    with cf.ThreadPoolExecutor(max_workers=workers) as ex:
        binding_obj = ex.submit(_compile_binding) if binding else None
        objs = list(ex.map(_compile, srcs))
    _link_library(objs)
    if binding_obj:
        _link_binding(binding_obj.result())
    if verbose:
        print(f"built {LIB_PATH} from {len(srcs)} sources{'' if binding else ', without the binding'}", file=sys.stderr)
    return LIB_PATH


if __name__ == "__main__":
    build()
