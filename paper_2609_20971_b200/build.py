"""Builds the C-ABI CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librbs_b200.so")
LIB_DEBUG = os.path.join(PKG, "librbs_b200_debug.so")   # the same sources with -DRBS_DEBUG: device-side index checks
SOURCES = ["rbs_api.cu", "rbs_tmap.cu", "rbs_stats.cu", "rbs_select.cu", "rbs_prefill.cu", "rbs_prefill_duo.cu", "rbs_union.cu", "rbs_box.cu", "rbs_varlen.cu",
           "rbs_extend.cu", "rbs_rope.cu", "rbs_decode.cu"]
NATIVE = os.path.join(PKG, "_native.so")                # marshalling of PyTorch's tensors, see csrc/rbs_torch.cpp
NATIVE_SOURCE = os.path.join(CSRC, "rbs_torch.cpp")
NATIVE_STAMP = os.path.join(PKG, "_native.stamp")       # the PyTorch and the Python that it was built against
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def needs_build(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))]
    deps += [os.path.join(ROOT, "include", "rbs.h"), os.path.join(ROOT, "include", "rbs_selftest.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def native_stamp() -> str | None:
    """What the marshalling module is bound to; None where PyTorch is missing or has no CUDA, and the module cannot be built."""
    try:
        import torch
    except ImportError:
        return None
    return f"torch {torch.__version__}, Python {sys.version_info.major}.{sys.version_info.minor}" if torch.version.cuda else None


def needs_native() -> bool:
    """Whether the module is missing, older than its source, or built against another PyTorch or Python."""
    deps = (NATIVE_SOURCE, os.path.join(ROOT, "include", "rbs.h"))
    if not os.path.exists(NATIVE) or not os.path.exists(NATIVE_STAMP) or any(os.path.getmtime(d) > os.path.getmtime(NATIVE) for d in deps):
        return True
    with open(NATIVE_STAMP) as f:
        return f.read() != native_stamp()


def build_native(force: bool = False) -> str:
    """Compiles the marshalling module with the host compiler against the installed PyTorch."""
    stamp = native_stamp()
    if stamp is None:
        raise RuntimeError("the marshalling module of the serving calls needs a PyTorch with CUDA")
    if not force and not needs_native():
        return NATIVE
    import sysconfig

    import torch
    base = os.path.join(os.path.dirname(torch.__file__))
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    system = [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"),
              sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-shared",
                    f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
                    *(x for p in system for x in ("-isystem", p)), NATIVE_SOURCE, "-o", NATIVE, "-L", os.path.join(base, "lib"),
                    "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"], check=True)
    with open(NATIVE_STAMP, "w") as f:
        f.write(stamp)
    return NATIVE


def build_library(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Compiles the sources (in parallel) and links the library; debug=True builds the checking variant.  The marshalling module is built
    along where the installed PyTorch allows; the library needs no PyTorch."""
    from concurrent.futures import ThreadPoolExecutor

    lib = LIB_DEBUG if debug else LIB
    if native_stamp() is not None:
        build_native(force)
    if not force and not needs_build(lib):
        return lib
    suffix = ".debug.o" if debug else ".o"
    extra = ["-DRBS_DEBUG"] if debug else []

    def compile_one(src: str) -> str:
        obj = os.path.join(CSRC, src.replace(".cu", suffix))
        cmd = [_nvcc(), *NVCC_FLAGS, *extra, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
               os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        subprocess.run(cmd, check=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    subprocess.run([_nvcc(), "-shared", "-o", lib, *objs, "-lcudart_static", "-ldl", "-lrt", "-lpthread"], check=True)
    return lib


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
