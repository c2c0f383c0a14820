"""Build the CAT W4A4 CUDA library (``libcatw4a4.so``) in-tree for sm_103a.

Every translation unit is compiled by ``nvcc`` in parallel, then linked into one shared library
next to this file.  The CUDA runtime is linked statically; the driver API (tensor-map encoding)
is reached through ``cudaGetDriverEntryPointByVersion``, so nothing links against libcuda.  The Python
calls of the microscaled operators (``_mx_calls``, an extension module of this interpreter on torch's C++ headers) link
against that library, which is there without them: where they do not build, the build says so and fails behind it.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libcatw4a4.so")
SOURCES = ["api.cu", "calib_cov.cu", "calib_cov_tc.cu", "act_quant.cu", "act_quant_tc.cu", "act_quant_few.cu", "gemm_tc.cu", "gemm_decode.cu", "gemm_decode_tc.cu", "sqnr.cu", "diag.cu", "quant_dp.cu", "gemm_dp.cu", "transform_dev.cu", "mx_quant.cu", "mx_gemm.cu", "mx_cache.cu", "mx_attention.cu", "mx_attention_tiles.cu", "transform_host.cpp"]
CALLS = os.path.join(HERE, "_mx_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-O3,-pthread", "-I", os.path.join(ROOT, "include")]


def nvcc() -> str:
    path = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(path):
        raise RuntimeError("nvcc not found")
    return path


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [nvcc(), *ARCH, *COMMON, "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose and src.endswith(".cu"):
        cmd.insert(1, "-Xptxas=-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{res.stderr}")
    if verbose and res.stderr:
        sys.stderr.write(res.stderr)
    return obj


def _run(cmd: list, what: str) -> None:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{res.stderr}")


def _compile_calls() -> str:
    import torch
    root = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    obj = os.path.join(BUILD, "mx_calls.o")
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-pthread", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          "-I", sysconfig.get_paths()["include"], "-I", root, "-I", cuda, "-c", os.path.join(CSRC, "mx_calls.cpp"), "-o", obj],
         "compiling mx_calls.cpp")
    return obj


def _link_calls(obj: str) -> None:
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = CALLS + ".tmp"
    _run(["g++", "-shared", "-pthread", "-o", tmp, obj, "-L", HERE, "-l:" + os.path.basename(LIB), "-L", libs, "-ltorch_python",
          "-ltorch_cpu", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN"], "linking _mx_calls")
    os.replace(tmp, CALLS)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        calls = ex.submit(_compile_calls)
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    tmp = LIB + ".tmp"
    cmd = [nvcc(), *ARCH, "-shared", "-Xcompiler", "-pthread", "-o", tmp, *objs]
    _run(cmd, "link")
    os.replace(tmp, LIB)
    _link_calls(calls.result())
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
