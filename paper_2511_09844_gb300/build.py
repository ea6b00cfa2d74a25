"""Build libsd2.so (the SD^2 C-ABI library) in-tree for sm_103a with nvcc.

Each translation unit under csrc/ is compiled in parallel to an object, then linked into
paper_2511_09844_gb300/_lib/libsd2.so. A rebuild happens only when a source or header is newer
than the library. No torch extension machinery is used: the library has a plain C ABI. Beside it
the compiled part of the Python binding (csrc/binding.cpp) is built with g++ against torch's headers; where that cannot
be done (no torch, no headers), the binding makes its calls through ctypes.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig
from importlib import metadata

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT_DIR = os.path.join(PKG, "_lib")
LIB = os.path.join(OUT_DIR, "libsd2.so")
SOURCES = ["engine.cu", "gemm_simt.cu", "gemm_tc.cu", "attention.cu", "norm.cu", "sampling.cu", "state.cu", "noalloc.cu", "chain.cu",
           "pages.cu", "prompt_attention.cu", "quantized_pages.cu", "quantized_attention.cu", "few_rows.cu",
           "quantized_tiles.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fno-strict-aliasing",
         "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include")]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _inputs():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h", ".cpp"))]
    files.append(os.path.join(ROOT, "include", "sd2.h"))
    files.append(os.path.abspath(__file__))
    return files


def binding_path():
    """The binding's compiled part for this Python and torch (one of another torch may load and not fit), None without torch."""
    try:
        version = metadata.version("torch")
    except metadata.PackageNotFoundError:
        return None
    return os.path.join(OUT_DIR, f"sd2_binding-{version}-{sys.implementation.cache_tag}.so")


def _failed(binding: str) -> str:
    """Stands in the place of a binding that could not be compiled, so that this is not tried at every build."""
    return binding + ".failed"


def is_stale() -> bool:
    made, binding = [LIB], binding_path()
    if binding is not None:
        made.append(binding if os.path.exists(binding) else _failed(binding))
    if not all(map(os.path.exists, made)):
        return True
    t = min(map(os.path.getmtime, made))
    return any(os.path.getmtime(f) > t for f in _inputs())


def _build_binding() -> None:
    """Compile binding.cpp if that can be done; the reason is reported if not."""
    binding = binding_path()
    if binding is None:
        return
    try:
        _compile_binding(binding)
        why = None
    except (ImportError, OSError, RuntimeError) as e:
        why = str(e)
        sys.stderr.write(f"binding.cpp is left out, calls go through ctypes: {why}\n")
    if why is None and os.path.exists(_failed(binding)):
        os.remove(_failed(binding))
    if why is not None:
        if os.path.exists(binding):          # (of older sources)
            os.remove(binding)
        with open(_failed(binding), "w") as f:
            f.write(why)


def _compile_binding(binding: str) -> None:
    import torch
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    dirs = [os.path.join(ROOT, "include"), os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
            os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    lib, tmp = os.path.join(home, "lib"), binding + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-I{d}" for d in dirs), os.path.join(CSRC, "binding.cpp"), "-o", tmp, f"-L{lib}", "-ltorch_python", "-ltorch",
           "-ltorch_cpu", "-lc10", "-lc10_cuda", f"-Wl,-rpath,{lib}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        raise RuntimeError("g++ failed\n" + r.stdout + r.stderr)
    os.replace(tmp, binding)


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    """Compile and link libsd2.so, and the binding where it can be; returns the library's path. Raises on any error of the
    library's."""
    if not force and not is_stale():
        return LIB
    os.makedirs(OUT_DIR, exist_ok=True)
    nvcc = _nvcc()
    objs = []

    def compile_one(src):
        obj = os.path.join(OUT_DIR, src.replace(".cu", ".o"))
        cmd = [nvcc, *ARCH, *FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or r.returncode:
            sys.stderr.write(r.stdout + r.stderr)
        if r.returncode:
            raise RuntimeError(f"nvcc failed on {src}")
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = ex.submit(_build_binding)
        objs = list(ex.map(compile_one, SOURCES))
        binding.result()
    tmp = LIB + ".tmp"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-lcudart_static", "-ldl", "-lrt", "-lpthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link of libsd2.so failed")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
