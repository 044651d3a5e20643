"""Build libseer.so in-tree with nvcc for sm_103a (no CMake, no setuptools).

Translation units compile in parallel into ``_build/`` and link into
``paper_2607_14557_gb300/libseer.so``.  The library links the shared CUDA
runtime so it shares one runtime instance with PyTorch in the same process.
``binding.cpp`` becomes the extension module ``_seer_binding`` beside it.
"""
from __future__ import annotations

import concurrent.futures
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libseer.so")
BINDING = os.path.join(PKG, "_seer_binding.so")
SOURCES = ["seer_api.cu", "tc_gemm.cu", "tc_attn.cu", "simt.cu", "aux_kernels.cu", "seer_noalloc.cu", "paged_api.cu",
           "paged.cu", "gqa_simt.cu", "tc_causal.cu", "tc_tree.cu", "rotary.cu", "mass.cu", "tc_mass.cu", "evict.cu"]
HEADERS = ["common.cuh", "kernels.h", "attn_schedule.cuh", "api.h", "paged.h", "budget.h", "mass_common.cuh", "attn_math.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _cuda_lib_dir(nv: str) -> str:
    return os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nv))), "lib64")


def _older(path: str, deps) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(p) > os.path.getmtime(path) for p in deps if os.path.exists(p))


def _lib_stale() -> bool:
    return _older(LIB, [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(ROOT, "include", "seer.h"), __file__])


def _binding_stale() -> bool:
    if _older(BINDING, [os.path.join(CSRC, "binding.cpp"), os.path.join(ROOT, "include", "seer.h"), __file__]):
        return True
    try:
        with open(os.path.join(BUILD, "binding.for")) as f:
            return f.read() != _binding_for()
    except OSError:
        return True


def _binding_for() -> str:
    """The interpreter and torch that the extension module is compiled against."""
    return f"python {sys.version} torch {importlib.metadata.version('torch')} at {os.path.dirname(importlib.util.find_spec('torch').origin)}"


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    """Compile and link what is older than its sources; return libseer.so's path.  Where the
    extension module cannot be compiled (no Python or torch headers, no host compiler), libseer.so is
    there all the same when the error is raised."""
    lib_stale, binding_stale = force or _lib_stale(), force or _binding_stale()
    if not lib_stale and not binding_stale:
        return LIB
    nv = nvcc()
    os.makedirs(BUILD, exist_ok=True)
    common = [nv, *ARCH, "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"),
              "--expt-relaxed-constexpr", *extra_flags]

    def compile_one(src: str) -> str:
        obj = os.path.join(BUILD, src.replace(".cu", ".o"))
        cmd = [*common, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            print(r.stdout + r.stderr)
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = ex.submit(_compile_binding, nv) if binding_stale else None
        if lib_stale:
            objs = list(ex.map(compile_one, SOURCES))
            tmp = LIB + ".tmp"
            libdir = _cuda_lib_dir(nv)
            _run([nv, *ARCH, "-shared", "-cudart", "shared", "-o", tmp, *objs, "-Xlinker", f"-rpath,{libdir}"], "link")
            os.replace(tmp, LIB)
    if binding is not None:
        _link_binding(binding.result())
    return LIB


def _run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")


def _compile_binding(nv: str) -> str:
    import torch

    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    obj = os.path.join(BUILD, "binding.o")
    _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          "-I", inc, "-I", os.path.join(inc, "torch", "csrc", "api", "include"), "-I", sysconfig.get_paths()["include"],
          "-I", os.path.join(os.path.dirname(_cuda_lib_dir(nv)), "include"), "-c", os.path.join(CSRC, "binding.cpp"), "-o", obj],
         "compiling binding.cpp")
    return obj


def _link_binding(obj: str) -> None:
    import torch

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = BINDING + ".tmp"
    _run([os.environ.get("CXX", "g++"), "-shared", "-o", tmp, obj, "-L", PKG, "-l:libseer.so", "-L", lib, "-ltorch_python", "-lc10_cuda",
          "-lc10", f"-Wl,-rpath,$ORIGIN:{lib}"], "linking the binding")
    os.replace(tmp, BINDING)
    with open(os.path.join(BUILD, "binding.for"), "w") as f:
        f.write(_binding_for())


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
