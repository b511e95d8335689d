"""Build libpmpe.so in-tree with nvcc for sm_103a (no cmake, no torch
extension machinery): each .cu under csrc/ compiles to an object in
parallel, then one shared-library link.  Beside it the Python module _ops
(csrc/bind_ops.cpp) with g++ against the headers of the installed PyTorch; the
library needs neither, and is there where that module cannot be built."""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libpmpe.so")
OPS_SRC, OPS_OUT = os.path.join(CSRC, "bind_ops.cpp"), os.path.join(PKG, "_ops.so")
BUILD_DIR = os.path.join(ROOT, "_build")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libpmpe")


def _flags():
    return ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall", "-Xcompiler", "-fvisibility=hidden",
                   "-I", os.path.join(ROOT, "include"), "--expt-relaxed-constexpr"]


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _ops_command():
    """The command that builds _ops.so, and what it is built for."""
    import torch
    cxx = shutil.which("g++") or "g++"
    home = os.path.dirname(torch.__file__)
    include = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
               os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))), "include"), sysconfig.get_paths()["include"]]
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-Wall", "-fvisibility=hidden", "-shared", f'-DPMPE_BUILT_FOR="{torch.__version__}"',
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include")]
    for d in include:
        cmd += ["-isystem", d]
    # PyTorch's libraries are in the process by the time the module is loaded
    cmd += [OPS_SRC, "-o", OPS_OUT + ".tmp", "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cuda", "-ltorch_cpu",
            "-lc10_cuda", "-lc10"]
    return cmd, f"{torch.__version__} {sys.version}\n"


def build(verbose: bool = False, force: bool = False, ptxas_info: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    nvcc = _nvcc()
    sources = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    headers = sorted(glob.glob(os.path.join(CSRC, "*.cuh"))) + [os.path.join(ROOT, "include", "pmpe.h")]
    objs = []
    jobs = []
    for src in sources:
        obj = os.path.join(BUILD_DIR, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if force or ptxas_info or _stale(obj, [src] + headers):
            cmd = [nvcc] + _flags() + (["-Xptxas", "-v"] if ptxas_info else []) + ["-c", src, "-o", obj]
            jobs.append(cmd)

    ops_cmd = ops_error = built_for = None
    stamp = os.path.join(BUILD_DIR, "_ops.txt")
    try:
        ops_cmd, built_for = _ops_command()
    except Exception as e:  # no PyTorch
        ops_error = repr(e)
    ops = force or _stale(OPS_OUT, [OPS_SRC, os.path.join(ROOT, "include", "pmpe.h")]) or not os.path.exists(stamp) or \
        open(stamp).read() != built_for
    if ops and ops_cmd:
        jobs.insert(0, ops_cmd)

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    with cf.ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 4))) as ex:
        for cmd, r in ex.map(run, jobs):
            if verbose or ptxas_info or r.returncode != 0:
                sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
            if r.returncode != 0:
                if cmd is not ops_cmd:
                    raise RuntimeError(f"nvcc failed on {cmd[-3]}")
                ops_error = f"{cmd[0]} returned {r.returncode}"
    if ops and not ops_error:
        os.replace(OPS_OUT + ".tmp", OPS_OUT)
        with open(stamp, "w") as f:
            f.write(built_for)
    if force or _stale(OUT, objs):
        cmd = [nvcc] + ARCH + ["-shared", "-o", OUT + ".tmp"] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
            raise RuntimeError("link of libpmpe.so failed")
        os.replace(OUT + ".tmp", OUT)
    if ops_error:
        if os.path.exists(OPS_OUT):  # of another source or another PyTorch
            os.remove(OPS_OUT)
        raise RuntimeError(f"building _ops.so failed ({ops_error}); libpmpe.so is built")
    return OUT


if __name__ == "__main__":
    build(verbose="-v" in sys.argv, force="-f" in sys.argv, ptxas_info="--ptxas" in sys.argv)
    print(OUT)
