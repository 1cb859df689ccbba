"""Builds libhalo.so (CUDA, sm_100a, nvcc) and _marshal.so (argument marshalling, g++ against torch's headers) in-tree.
`python -m paper_2601_11676_b200.build [--force] [-v]`."""
from __future__ import annotations

import os
import subprocess
import sys
import warnings
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libhalo.so")
MARSHAL_SRC = os.path.join(PKG, "csrc_py", "marshal.cpp")
MARSHAL = os.path.join(PKG, "_marshal.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps_mtime() -> float:
    hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    hdrs.append(os.path.join(ROOT, "include", "halo.h"))
    return max(os.path.getmtime(p) for p in hdrs)


def marshal_made_for() -> str:
    """What _marshal.so depends on beside its source; compiled into it and compared when it is loaded."""
    import torch
    return f"torch {torch.__version__}, python {sys.version_info.major}.{sys.version_info.minor}"


def build_marshal(force: bool = False) -> str:
    """_marshal.so; rebuilt when its source, halo.h or the torch it was built against changed."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension
    stamp = os.path.join(OBJ, "marshal.torch")
    made_with = f"{torch.__version__} {torch.__file__} {sys.version}"
    newest = max(os.path.getmtime(p) for p in (MARSHAL_SRC, os.path.join(ROOT, "include", "halo.h")))
    fresh = os.path.exists(MARSHAL) and os.path.getmtime(MARSHAL) >= newest and os.path.exists(stamp) and \
        open(stamp).read() == made_with
    if fresh and not force:
        return MARSHAL
    lib_dir = os.path.join(os.path.dirname(torch.__file__), "lib")
    includes = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], "/usr/local/cuda/include",
                                                os.path.join(ROOT, "include")]
    tmp = MARSHAL + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DMARSHAL_MADE_FOR="{marshal_made_for()}"',
           *(f"-I{p}" for p in includes), MARSHAL_SRC, "-o", tmp, f"-L{lib_dir}", f"-Wl,-rpath,{lib_dir}", "-lc10", "-lc10_cuda",
           "-ltorch_cpu", "-ltorch", "-ltorch_python"]
    p = subprocess.run(cmd, capture_output=True, text=True)
    if p.returncode != 0:
        raise RuntimeError("g++ failed: " + " ".join(cmd) + "\n" + p.stdout + p.stderr)
    os.replace(tmp, MARSHAL)
    with open(stamp, "w") as f:
        f.write(made_with)
    return MARSHAL


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    hdr_time = _deps_mtime()
    jobs = []
    objs = []
    for src in sources():
        obj = os.path.join(OBJ, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        stale = force or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(src), hdr_time)
        if stale:
            cmd = [_nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []), "-c", src, "-o", obj]
            jobs.append(cmd)

    def run(cmd):
        p = subprocess.run(cmd, capture_output=True, text=True)
        if p.returncode != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd) + "\n" + p.stdout + p.stderr)
        return p.stderr

    if jobs:
        with ThreadPoolExecutor(max_workers=min(8, len(jobs))) as ex:
            for log in ex.map(run, jobs):
                if verbose and log:
                    print(log, file=sys.stderr)
    if jobs or not os.path.exists(LIB):
        tmp = LIB + f".tmp{os.getpid()}"
        run([_nvcc(), "-shared", "-o", tmp, *objs, "-lcudart"])
        os.replace(tmp, LIB)
    try:
        build_marshal(force)
    except Exception as e:     # no g++, no headers of Python or torch: the library is complete without it
        if os.path.exists(MARSHAL):
            os.remove(MARSHAL)     # of an older source
        warnings.warn(f"{MARSHAL} was not built, so the entry points of a batched token step (halo_paged_*, halo_norm_glue, "
                      f"halo_*_mx4) cannot be called from Python: {e}")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
