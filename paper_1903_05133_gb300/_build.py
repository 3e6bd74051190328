"""Compile the CUDA C-ABI library ``libhier_avg.so`` in-tree for sm_103a, and the Python
binding's host module ``_host.so``.

Each translation unit is compiled by nvcc in parallel, then linked with the
static CUDA runtime into one shared library next to this file.  Arithmetic flags
are explicit: no fast-math, IEEE division and square root, subnormals kept.
The host module is compiled by g++ against Python's and PyTorch's headers, beside them.  Where that is not
possible the library is built all the same: the C ABI needs neither, and _lib.host() raises where the module
is missing.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "libhier_avg.so")
HOST_PATH = os.path.join(HERE, "_host.so")

SOURCES = ["hier_avg_api.cu", "avg_kernels.cu", "step_tc.cu", "step_head.cu", "step_fp32.cu",
           "op_grouped.cu", "op_logprobs.cu", "op_adamw.cu", "op_route.cu", "op_rows.cu", "op_norm.cu",
           "op_verify.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-ftz=false",
          "-prec-div=true", "-prec-sqrt=true", f"-I{INCLUDE}", f"-I{CSRC}"]
EXTRA = {"avg_kernels.cu": ["-fmad=false"], "op_adamw.cu": ["-fmad=false"]}


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libhier_avg.so")


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("command failed:\n" + " ".join(cmd) + "\n" + r.stdout)
    return r.stdout


def _cuda_include() -> str:
    return os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(_nvcc()))), "include")


def _host_command(out: str):
    """g++ on csrc/host.cpp; the libraries are those that ``import torch`` has loaded."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        raise RuntimeError("PyTorch not found")
    torch = spec.submodule_search_locations[0]
    inc, lib = os.path.join(torch, "include"), os.path.join(torch, "lib")
    return [os.environ.get("CXX") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-o", out,
            os.path.join(CSRC, "host.cpp"), f"-I{sysconfig.get_paths()['include']}", f"-isystem{inc}",
            f"-isystem{os.path.join(inc, 'torch', 'csrc', 'api', 'include')}", f"-L{lib}", f"-isystem{_cuda_include()}",
            "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def _compile_host():
    """What stands in the way of the host module, or None where it is compiled (to HOST_PATH.tmp)."""
    try:
        _run(_host_command(HOST_PATH + ".tmp"))
    except (RuntimeError, OSError) as e:
        return e


def build(verbose: bool = False, ptxas_info: bool = False) -> str:
    nvcc = _nvcc()
    os.makedirs(BUILD_DIR, exist_ok=True)
    objs, cmds = [], []
    for src in SOURCES:
        obj = os.path.join(BUILD_DIR, src.replace(".cu", ".o"))
        cmd = [nvcc, *ARCH, *COMMON, *EXTRA.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
        if ptxas_info:
            cmd += ["-Xptxas", "-v"]
        objs.append(obj)
        cmds.append(cmd)
    with ThreadPoolExecutor(max_workers=len(cmds) + 1) as ex:
        host = ex.submit(_compile_host)
        outs = list(ex.map(_run, cmds))
    if verbose or ptxas_info:
        for o in outs:
            sys.stdout.write(o)
    tmp = LIB_PATH + ".tmp"
    _run([nvcc, *ARCH, "-shared", "--cudart", "static", "-o", tmp, *objs])
    os.replace(tmp, LIB_PATH)
    missing = host.result()
    if missing is None:
        os.replace(HOST_PATH + ".tmp", HOST_PATH)
    else:
        if os.path.exists(HOST_PATH):           # of another build
            os.remove(HOST_PATH)
        sys.stderr.write(f"{LIB_PATH} is built, the Python binding's host module is not, which the routing, row, norm and "
                         f"draft operators of the binding need: {missing}\n")
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True, ptxas_info="-v" in sys.argv))
