"""Build the C-ABI library libspecflash_verify.so for sm_103a, in-tree.

Each .cu file under csrc/ is compiled separately (in parallel) with
``nvcc -gencode arch=compute_103a,code=sm_103a -O3 -lineinfo`` and linked
with the static CUDA runtime into ``_build/libspecflash_verify.so``, so the
library needs only the NVIDIA driver at run time.  Rebuilds only when a
source or header is newer than the library.

csrc/layer_calls.cpp (the decoder-layer operators' calls from Python without the
detour through ctypes) is compiled beside it with g++ and torch's headers into
``_build/_layer_calls.<Python>.<torch>.so``; where that fails, the binding does without.
"""
from __future__ import annotations

import glob
import os
import re
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(BUILD, "libspecflash_verify.so")
CALLS_SOURCE = os.path.join(CSRC, "layer_calls.cpp")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-O2",
              "--expt-relaxed-constexpr", "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build the library")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _inputs():
    return sources() + glob.glob(os.path.join(CSRC, "*.h")) + \
        glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))


def up_to_date() -> bool:
    if not os.path.exists(LIB):
        return False
    t = os.path.getmtime(LIB)
    return all(os.path.getmtime(f) <= t for f in _inputs())


def calls_path() -> str:
    """Where _layer_calls is for the Python and the torch that run: torch's inline
    accessors are compiled into it, so one that was built for another torch may load
    and look at tensors through the wrong offsets."""
    import torch
    key = f"{sysconfig.get_config_var('SOABI')}.torch-{torch.__version__}-abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}"
    return os.path.join(BUILD, f"_layer_calls.{re.sub('[^A-Za-z0-9.+-]', '_', key)}.so")


def build_calls(force: bool = False) -> str | None:
    """Compile _layer_calls against the installed torch; its path, or None where that
    is not possible (the reason goes to stderr, and to a file beside it, so that the
    same source is not tried again)."""
    header = os.path.join(INCLUDE, "specflash_verify.h")
    newest = max(os.path.getmtime(CALLS_SOURCE), os.path.getmtime(header))
    try:
        path = calls_path()
    except (ImportError, AttributeError) as e:
        print(f"_layer_calls is not built: {e}", file=sys.stderr)
        return None
    failed = path + ".failed"
    if not force:
        if os.path.exists(path) and os.path.getmtime(path) >= newest:
            return path
        if os.path.exists(failed) and os.path.getmtime(failed) >= newest:
            return None
    try:
        import torch
        root = os.path.join(os.path.dirname(torch.__file__))
        inc = os.path.join(root, "include")
        lib = os.path.join(root, "lib")
        cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
        tmp = path + f".{os.getpid()}.tmp"
        cmd = ["g++", "-O2", "-shared", "-fPIC", "-std=c++17", "-fvisibility=hidden",
               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE,
               "-I", sysconfig.get_paths()["include"], "-isystem", cuda, "-isystem", inc,
               "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"), CALLS_SOURCE, "-o", tmp,
               "-L", lib, "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda", f"-Wl,-rpath,{lib}"]
        r = subprocess.run(cmd, capture_output=True, text=True)
    except (ImportError, AttributeError, OSError) as e:
        print(f"_layer_calls is not built: {e}", file=sys.stderr)
        return None
    if r.returncode != 0:
        print(f"_layer_calls is not built:\n{r.stderr[-2000:]}", file=sys.stderr)
        with open(failed, "w") as f:
            f.write(r.stderr)
        return None
    os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    os.makedirs(BUILD, exist_ok=True)
    if not force and up_to_date():
        build_calls()
        return LIB
    nvcc = _nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc, *ARCH, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout + r.stderr, flush=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        calls = ex.submit(build_calls, force)
        objs = list(ex.map(compile_one, sources()))
        calls.result()
    tmp = LIB + f".{os.getpid()}.tmp"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    flags = [a for a in sys.argv[1:] if a.startswith("-")]
    print(build(force=True, verbose=True, extra_flags=flags))
