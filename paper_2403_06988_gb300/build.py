"""Builds libdomino.so in-tree with nvcc for sm_103a (GB300).

Twelve translation units (host.cpp: C ABI and loaders; kernels.cu, rows.cu, logits.cu,
loss.cu, loss_few.cu, distill.cu, embed.cu, norm.cu, quantize8.cu, logits8.cu and penalized.cu:
kernels) are compiled in parallel and linked into paper_2403_06988_gb300/libdomino.so.
Objects go to paper_2403_06988_gb300/_build/.

csrc/calls.cpp becomes the Python extension _loss_calls.so beside it (g++, against the
installed torch's headers and libraries; built again for another torch or Python).  Without
a CUDA build of torch the library is built alone.

build(debug=True) makes libdomino_debug.so instead (objects in _build_debug/),
compiled with -DDOMINO_DEBUG: every transition-table lookup checks its state,
class and entry against the table's bounds and reports a violation in the
device error word (DOMINO_DEVERR_INTERNAL) instead of reading outside it.  The
binding loads it when DOMINO_DEBUG_LIB=1 is set in the environment.
"""
from __future__ import annotations

import concurrent.futures
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdomino.so")
LIB_DEBUG = os.path.join(PKG, "libdomino_debug.so")
CALLS = os.path.join(PKG, "_loss_calls.so")
SOURCES = ["host.cpp", "kernels.cu", "rows.cu", "logits.cu", "loss.cu", "loss_few.cu", "distill.cu", "embed.cu",
           "norm.cu", "quantize8.cu", "logits8.cu", "penalized.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libdomino.so")
    return exe


def _inputs():
    files = [os.path.join(CSRC, f) for f in SOURCES]
    files += [os.path.join(CSRC, f) for f in ("domino_internal.h", "walk_common.cuh", "decode.cuh", "loss.h", "norm.h", "tcgen05.cuh",
                                              "tensor_map.h", "bf16_rows.cuh", "values8.cuh")]
    files.append(os.path.join(INCLUDE, "domino.h"))
    return files


def up_to_date(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return False
    t = os.path.getmtime(lib)
    return all(os.path.getmtime(f) <= t for f in _inputs())


def _torch():
    """The folder of the installed torch if it is a CUDA build (not imported), else None."""
    spec = importlib.util.find_spec("torch")
    folder = spec and spec.submodule_search_locations and spec.submodule_search_locations[0]
    return folder if folder and os.path.exists(os.path.join(folder, "lib", "libc10_cuda.so")) else None


def _torch_version(folder) -> str:
    with open(os.path.join(folder, "version.py")) as f:
        return f.read()


def _calls_for(folder) -> str:
    """What the extension is built for: it unpacks this torch's objects in this Python."""
    return "\n".join((sysconfig.get_config_var("SOABI") or "", folder, _torch_version(folder)))


def calls_built_for_another() -> bool:
    """Whether _loss_calls.so is known to be built for another torch or Python than the installed one."""
    folder, stamp = _torch(), CALLS + ".for"
    if not folder:
        return True
    if not os.path.exists(stamp):
        return False
    with open(stamp) as f:
        return f.read() != _calls_for(folder)


def calls_up_to_date() -> bool:
    """Whether _loss_calls.so is there, built from its source for the installed torch."""
    src = [os.path.join(CSRC, "calls.cpp"), os.path.join(INCLUDE, "domino.h")]
    return (os.path.exists(CALLS) and os.path.exists(CALLS + ".for") and not calls_built_for_another() and
            all(os.path.getmtime(f) <= os.path.getmtime(CALLS) for f in src))


def build_calls(force: bool = False):
    """The Python extension _loss_calls.so (None without a CUDA build of torch)."""
    folder = _torch()
    if not folder:
        print("no CUDA build of torch is installed: libdomino.so is built without the Python calls of the losses and the "
              "embedding", file=sys.stderr)
        return None
    if not force and calls_up_to_date():
        return CALLS
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    lib = os.path.join(folder, "lib")
    tmp = CALLS + f".tmp{os.getpid()}"
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", os.path.join(CSRC, "calls.cpp"), "-o", tmp,
           "-I", INCLUDE, "-I", os.path.join(folder, "include"), "-I", sysconfig.get_paths()["include"],
           "-I", os.path.join(cuda, "include"), "-L", lib, f"-Wl,-rpath,{lib}", "-ltorch_python", "-ltorch_cpu",
           "-lc10_cuda", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for calls.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, CALLS)
    with open(tmp, "w") as f:
        f.write(_calls_for(folder))
    os.replace(tmp, CALLS + ".for")
    return CALLS


def build(force: bool = False, verbose: bool = False, extra_flags=(), debug: bool = False) -> str:
    with concurrent.futures.ThreadPoolExecutor(1) as calls:   # beside the kernels
        done = calls.submit(build_calls, force)
        lib = _build_library(force, verbose, extra_flags, debug)
        done.result()
    return lib


def _build_library(force, verbose, extra_flags, debug) -> str:
    lib = LIB_DEBUG if debug else LIB
    bdir = BUILD + "_debug" if debug else BUILD
    if not force and up_to_date(lib):
        return lib
    os.makedirs(bdir, exist_ok=True)
    exe = nvcc()
    common = ["-O3", "-std=c++17", *ARCH, "-lineinfo", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC,
              *(["-DDOMINO_DEBUG"] if debug else []), *extra_flags]
    if verbose:
        common += ["-Xptxas", "-v"]

    def compile_one(src):
        obj = os.path.join(bdir, os.path.splitext(src)[0] + ".o")
        cmd = [exe, *common, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        return obj, r.stderr

    with concurrent.futures.ThreadPoolExecutor(len(SOURCES)) as ex:
        results = list(ex.map(compile_one, SOURCES))
    if verbose:
        for _, log in results:
            print(log)
    tmp = lib + f".tmp{os.getpid()}"
    cmd = [exe, "-shared", *ARCH, "-o", tmp, *[o for o, _ in results]]   # cudart linked statically
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
