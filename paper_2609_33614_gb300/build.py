"""Build libeat.so in-tree for sm_103a (GB300): one nvcc call per translation unit, in parallel,
then one link; and beside it _eatops.so, the Python binding of the operators on torch tensors.
Rebuilds only when a source, header or flag changed (content hash stamp)."""
from __future__ import annotations

import concurrent.futures as cf
import glob
import hashlib
import os
import shutil
import subprocess
import sysconfig
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libeat.so")
BINDING = os.path.join(PKG, "_eatops.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xptxas", "-warn-spills",
         "-I", os.path.join(ROOT, "include")]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", shutil.which("nvcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stamp() -> str:
    h = hashlib.sha256()
    files = _sources() + sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + \
        [os.path.join(ROOT, "include", "eat.h")]
    for f in files:
        h.update(f.encode())
        with open(f, "rb") as fh:
            h.update(fh.read())
    h.update(" ".join(ARCH + FLAGS).encode())
    return h.hexdigest()


# Sources that define the tensor-core FFN kernels: a DRAM-traffic capture of those kernels stays
# valid while these files are unchanged (the rest of the library does not touch their code).
FFN_SOURCES = ("ffn_tc.cu", "ffn_tc.cuh")


def _strip_comments(src: str) -> str:
    """C/C++ source without its // and /* */ comments (string and character literals kept)."""
    out, i, n = [], 0, len(src)
    while i < n:
        c = src[i]
        if c in "\"'":
            j = i + 1
            while j < n and src[j] != c:
                j += 2 if src[j] == "\\" else 1
            out.append(src[i:j + 1])
            i = j + 1
        elif src.startswith("//", i):
            j = src.find("\n", i)
            i = n if j < 0 else j
        elif src.startswith("/*", i):
            j = src.find("*/", i + 2)
            i = n if j < 0 else j + 2
        else:
            out.append(c)
            i += 1
    return "".join(out)


def ffn_source_hash() -> str:
    """Hash of the FFN kernel sources (comments removed, whitespace runs as one space: edits of
    comments and layout keep it) and the compile flags, independent of where the repository lives
    (the include path enters relative to the repository root)."""
    h = hashlib.sha256()
    for name in FFN_SOURCES:
        with open(os.path.join(CSRC, name), encoding="utf-8") as fh:
            h.update(name.encode())
            h.update(" ".join(_strip_comments(fh.read()).split()).encode())
    flags = [os.path.relpath(f, ROOT) if os.path.isabs(f) else f for f in ARCH + FLAGS]
    h.update(" ".join(flags).encode())
    return h.hexdigest()


def _binding_needs():
    """(include directories, library directory, compiler) of the binding; RuntimeError with what is
    missing.  libeat.so needs none of it."""
    try:
        import torch
    except ImportError as e:
        raise RuntimeError(f"torch cannot be imported ({e})") from None
    root = os.path.dirname(torch.__file__)
    python = sysconfig.get_paths()["include"]
    inc = [os.path.join(ROOT, "include"), os.path.join(root, "include"),
           os.path.join(root, "include", "torch", "csrc", "api", "include"),
           os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))), "include"),
           python]
    for f in (os.path.join(root, "include", "ATen", "core", "Tensor.h"),
              os.path.join(python, "Python.h")):
        if not os.path.exists(f):
            raise RuntimeError(f"{f} is missing")
    cxx = os.environ.get("CXX", "g++")
    if not shutil.which(cxx.split()[0]):
        raise RuntimeError(f"no C++ compiler ({cxx})")
    return inc, os.path.join(root, "lib"), cxx.split()


def _build_binding(force: bool = False) -> str:
    """Compile and link _eatops.so against the installed torch and libeat.so (found beside it)."""
    inc, lib, cxx = _binding_needs()
    import torch
    src = os.path.join(CSRC, "binding.cpp")
    flags = ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    h = hashlib.sha256(" ".join(flags + inc + [torch.__version__]).encode())
    for f in (src, os.path.join(ROOT, "include", "eat.h")):
        with open(f, "rb") as fh:
            h.update(fh.read())
    stamp_file = os.path.join(BUILD, "eatops.stamp")
    if not force and os.path.exists(BINDING) and os.path.exists(stamp_file):
        with open(stamp_file) as fh:
            if fh.read().strip() == h.hexdigest():
                return BINDING
    obj = os.path.join(BUILD, "binding.o")
    tmp = BINDING + ".tmp"
    # (torch's libraries are loaded before it; libeat.so is found in its own directory)
    libs = ["-L" + lib, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python",
            "-L" + PKG, "-l:libeat.so", "-Wl,-rpath,$ORIGIN"]
    for cmd in (cxx + flags + ["-I" + i for i in inc] + ["-c", src, "-o", obj],
                cxx + ["-shared", "-o", tmp, obj] + libs):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"{' '.join(cmd[:2])} failed on {src}:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING)
    with open(stamp_file, "w") as fh:
        fh.write(h.hexdigest())
    return BINDING


def build(verbose: bool = False, force: bool = False) -> str:
    """Compile and link libeat.so and its Python binding; returns the library's path.  Where torch, its
    headers, Python's or a C++ compiler are missing, the library is built alone, with a warning: the
    C ABI and the ctypes functions work, and the functions of torch tensors say what they lack."""
    path = _build_library(verbose, force)
    try:
        _binding_needs()
    except RuntimeError as e:
        if os.path.exists(BINDING):
            os.remove(BINDING)  # of another library, as a rule
        warnings.warn(f"_eatops.so is not built: {e}")
        return path
    _build_binding(force)
    return path


def _build_library(verbose: bool, force: bool) -> str:
    os.makedirs(BUILD, exist_ok=True)
    stamp_file = os.path.join(BUILD, "libeat.stamp")
    stamp = _stamp()
    if not force and os.path.exists(LIB) and os.path.exists(stamp_file):
        with open(stamp_file) as fh:
            if fh.read().strip() == stamp:
                return LIB
    nvcc = _nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        cmd = [nvcc] + ARCH + FLAGS + ["-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout + r.stderr)
        return obj

    srcs = _sources()
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs), os.cpu_count() or 4)) as ex:
        objs = list(ex.map(compile_one, srcs))
    tmp = LIB + ".tmp"
    cmd = [nvcc] + ARCH + ["-shared", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    with open(stamp_file, "w") as fh:
        fh.write(stamp)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, force=True))
