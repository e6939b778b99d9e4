"""Builds libembedpart.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _head.so beside it."""
from __future__ import annotations

import importlib.metadata
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libembedpart.so")
OBJ_DEBUG = os.path.join(PKG, "_build_debug")
LIB_DEBUG = os.path.join(PKG, "libembedpart_debug.so")   # the bounds-checked build (-DEP_DEBUG)

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


HEAD = os.path.join(PKG, "_head.so")                      # tensor marshalling of the partition head's operators


def head_commands():
    """(compile, link) of _head.so: host code against torch's own headers and libraries."""
    import torch
    base = os.path.dirname(torch.__file__)
    lib = os.path.join(base, "lib")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    obj = os.path.join(OBJ, "head_binding.o")
    inc = [x for d in [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include"), sysconfig.get_paths()["include"],
                       os.path.join(ROOT, "include")] for x in ("-isystem", d)]
    cxx = os.environ.get("CXX", "g++")
    return ([cxx, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
             *inc, "-c", os.path.join(CSRC, "head_binding.cpp"), "-o", obj],
            [cxx, "-shared", obj, "-L", lib, "-Wl,-rpath," + lib, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch",
             "-ltorch_python", "-o"])


def head_stamp():
    """What _head.so is built for, besides its sources: another torch or Python has another binary interface."""
    return "torch %s, python %s, %s" % (importlib.metadata.version("torch"), sysconfig.get_config_var("SOABI"), os.environ.get("CXX", "g++"))


def sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def _newest_header():
    hs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    hs.append(os.path.join(ROOT, "include", "embedpart.h"))
    return max(os.path.getmtime(h) for h in hs)


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Builds the library; debug = the bounds-checked variant (also chosen by EP_DEBUG=1 in the environment)."""
    debug = debug or os.environ.get("EP_DEBUG", "") == "1"
    nvcc = os.environ.get("NVCC", "nvcc")
    OBJ, LIB = (OBJ_DEBUG, LIB_DEBUG) if debug else (globals()["OBJ"], globals()["LIB"])
    extra = ["-DEP_DEBUG"] if debug else []
    os.makedirs(OBJ, exist_ok=True)
    hdr = _newest_header()
    jobs = []
    objs = []
    for f in sources():
        src = os.path.join(CSRC, f)
        obj = os.path.join(OBJ, f[:-3] + ".o")
        objs.append(obj)
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(src), hdr):
            cmd = [nvcc, *NVCC_FLAGS, *extra, *os.environ.get("EP_NVCC_EXTRA", "").split(), "-c", src, "-o", obj]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
            jobs.append(cmd)

    # the head's extension, the same beside either library
    mark, stamp = os.path.join(globals()["OBJ"], "head_binding.stamp"), head_stamp()
    head_new = force or not os.path.exists(HEAD) or os.path.getmtime(HEAD) < max(os.path.getmtime(os.path.join(CSRC, "head_binding.cpp")), hdr)
    if not head_new:
        head_new = not os.path.exists(mark) or open(mark).read() != stamp
    head_jobs = [head_commands()[0]] if head_new else []
    os.makedirs(globals()["OBJ"], exist_ok=True)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("compiler failed: %s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
        return r.stderr

    with ThreadPoolExecutor(max_workers=max(1, min(8, len(jobs + head_jobs)))) as ex:
        for log in ex.map(run, jobs + head_jobs):
            if verbose and log:
                print(log, file=sys.stderr)
    if jobs or not os.path.exists(LIB):
        tmp = LIB + ".tmp.%d" % os.getpid()
        run([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", tmp, *objs, "-lcudart_static",
             "-ldl", "-lrt", "-lpthread"])
        os.replace(tmp, LIB)
    if head_new:
        tmp = HEAD + ".tmp.%d" % os.getpid()
        run([*head_commands()[1], tmp])
        os.replace(tmp, HEAD)
        with open(mark, "w") as f:
            f.write(stamp)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
