"""Builds libmoara.so in-tree with nvcc for sm_103a.

Each translation unit under csrc/ compiles to an object in _build/ (in
parallel); the objects link into paper_2609_15037_gb300/libmoara.so.  A unit is
recompiled only when it or a header is newer than its object.  host.cpp, the
Python module that reads tensors, is built apart from it against torch's headers into paper_2609_15037_gb300/_host.so.
"""

from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import platform
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT_DIR = os.path.join(PKG, "_build", platform.machine())
LIB = os.path.join(PKG, "libmoara.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall",
          "-I", os.path.join(ROOT, "include")]


def _nvcc():
    exe = shutil.which("nvcc")
    if exe is None:
        cand = "/usr/local/cuda/bin/nvcc"
        if os.path.exists(cand):
            return cand
        raise RuntimeError("nvcc not found")
    return exe


HOST_SRC = os.path.join(CSRC, "host.cpp")
HOST = os.path.join(PKG, "_host.so")


def _sources():
    return sorted(s for s in glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp"))
                  if s != HOST_SRC)


def _headers():
    return glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(ROOT, "include", "*.h"))


def _compile(src, verbose_ptxas=False):
    obj = os.path.join(OUT_DIR, os.path.basename(src) + ".o")
    newest = max([os.path.getmtime(src)] + [os.path.getmtime(h) for h in _headers()])
    if os.path.exists(obj) and os.path.getmtime(obj) >= newest and not verbose_ptxas:
        return obj, ""
    cmd = [_nvcc()] + ARCH + COMMON + ["-c", src, "-o", obj]
    if verbose_ptxas and src.endswith(".cu"):
        cmd += ["-Xptxas", "-v"]
    p = subprocess.run(cmd, capture_output=True, text=True)
    if p.returncode != 0:
        raise RuntimeError(f"nvcc failed for {os.path.basename(src)}:\n{p.stdout}\n{p.stderr}")
    return obj, p.stderr


def _identity(path):
    """Which file is at `path`: the libraries lie beside the sources, where a build on another
    machine replaces them."""
    s = os.stat(path)
    return f"{path} {s.st_size} {s.st_mtime_ns}"


def _host_command(out):
    import torch
    root = os.path.dirname(torch.__file__)
    return [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-isystem", os.path.join(root, "include"),
            "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
            "-isystem", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"), HOST_SRC, "-o", out,
            "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]


def _host_key():
    """What _host.so was built from, by what and on which machine, and which file it is."""
    import torch
    return "\n".join([platform.machine(), torch.__version__, sys.version, *_host_command(HOST),
                      *(str(os.stat(f).st_mtime_ns) for f in (HOST_SRC, os.path.join(ROOT, "include", "moara.h"))),
                      _identity(HOST)])


def _build_host():
    """_host.so: again when its key is another one."""
    stamp = os.path.join(OUT_DIR, "host.stamp")
    if os.path.exists(HOST) and os.path.exists(stamp):
        with open(stamp) as f:
            if f.read() == _host_key():
                return
    tmp = HOST + ".tmp"
    p = subprocess.run(_host_command(tmp), capture_output=True, text=True)
    if p.returncode != 0:
        raise RuntimeError(f"g++ failed for host.cpp:\n{p.stdout}\n{p.stderr}")
    os.replace(tmp, HOST)
    with open(stamp, "w") as f:
        f.write(_host_key())


def build(verbose_ptxas=False, jobs=None):
    """Compile every CUDA/C++ unit for sm_103a, link libmoara.so, and build _host.so."""
    os.makedirs(OUT_DIR, exist_ok=True)
    srcs = _sources()
    with cf.ThreadPoolExecutor(max_workers=jobs or min(8, len(srcs) + 1)) as ex:
        host = ex.submit(_build_host)
        results = list(ex.map(lambda s: _compile(s, verbose_ptxas), srcs))
        host.result()
    objs = [r[0] for r in results]
    if verbose_ptxas:
        for _, log in results:
            if log:
                sys.stderr.write(log)
    newest = max(os.path.getmtime(o) for o in objs)
    stamp = os.path.join(OUT_DIR, "lib.stamp")
    fresh = (os.path.exists(LIB) and os.path.exists(stamp) and
             os.path.getmtime(LIB) >= newest and open(stamp).read() == _identity(LIB))
    if not fresh:
        tmp = LIB + ".tmp"
        cmd = [_nvcc()] + ARCH + ["-shared", "-o", tmp] + objs + ["-lcudart"]
        p = subprocess.run(cmd, capture_output=True, text=True)
        if p.returncode != 0:
            raise RuntimeError(f"link failed:\n{p.stdout}\n{p.stderr}")
        os.replace(tmp, LIB)
        with open(stamp, "w") as f:
            f.write(_identity(LIB))
    return LIB


if __name__ == "__main__":
    print(build(verbose_ptxas="-v" in sys.argv))
