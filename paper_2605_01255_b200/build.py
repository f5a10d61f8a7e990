"""Builds libacx.so (sm_100a) in-tree with nvcc, and the Python side's argument checks with g++ against the installed torch.
`python -m paper_2605_01255_b200.build [--force] [--library-only]`; the library alone, all that users of the C ABI need, is
built without torch's and Python's headers."""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libacx.so")
HOST_SRC = os.path.join(CSRC, "host_calls.cpp")
HOST_PATH = os.path.join(HERE, "_acx_host.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--fmad=true",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: cannot build libacx.so")


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _headers():
    hs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    hs.append(os.path.join(os.path.dirname(HERE), "include", "acx.h"))
    return hs


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _host_job(force: bool):
    """The command that builds the host module against the installed torch, or None where it is up to date."""
    import torch

    if not force and not _stale(HOST_PATH, [HOST_SRC, _headers()[-1], torch.version.__file__]):
        return None
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    # g++ of the path, as nvcc takes it: torch and this module have to share one libstdc++
    return [shutil.which("g++") or os.environ.get("CXX") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
            *("-I" + d for d in (sysconfig.get_paths()["include"], os.path.join(home, "include"),
                                 os.path.join(home, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include"))),
            HOST_SRC, "-o", HOST_PATH, "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def build(force: bool = False, verbose: bool = False, extra_flags=(), library_only: bool = False) -> str:
    """Compile every .cu under csrc/, link libacx.so next to this file and build the host module.  Returns the library path.  A host
    module that cannot be built is an error that is raised once the library is in place."""
    nvcc = _nvcc()
    os.makedirs(OBJ_DIR, exist_ok=True)
    headers = _headers()
    jobs = []
    objs = []
    for src in _sources():
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if force or _stale(obj, [src] + headers):
            jobs.append([nvcc, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", obj])
    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("build failed:\n%s\n%s\n%s" % (" ".join(cmd), r.stdout, r.stderr))
        if verbose and (r.stdout or r.stderr):
            print(r.stdout, r.stderr, flush=True)

    def run_host():
        job = _host_job(force)
        if job:
            run(job)

    with concurrent.futures.ThreadPoolExecutor(max_workers=max(1, min(8, len(jobs) + 1))) as ex:
        host = None if library_only else ex.submit(run_host)
        list(ex.map(run, jobs))
    if jobs or force or _stale(LIB_PATH, objs):
        run([nvcc, "-shared", "-o", LIB_PATH, *objs])
    if host and host.exception():
        raise RuntimeError("%s is built; the argument checks of the Python binding (%s) are not" % (LIB_PATH, HOST_PATH)) from host.exception()
    return LIB_PATH


if __name__ == "__main__":
    extra = ["-Xptxas", "-v"] if "--ptxas" in sys.argv else []
    print(build(force="--force" in sys.argv, verbose=True, extra_flags=extra, library_only="--library-only" in sys.argv))
