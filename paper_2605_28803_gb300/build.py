"""Build libqvla.so in-tree for sm_103a (GB300) with nvcc: one object per source, compiled in
parallel, then linked into paper_2605_28803_gb300/libqvla.so.  The CUDA runtime is linked
statically so the library needs nothing on LD_LIBRARY_PATH.  Beside it _calls, the part of the
Python binding that is compiled (csrc/calls.c; it finds libqvla.so in its own folder), under the tag
of the interpreter that it is compiled for."""

from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libqvla.so")
CALLS = os.path.join(PKG, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
INCLUDE = os.path.join(os.path.dirname(PKG), "include")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
SOURCES = ["rotate_quant_f16.cu", "rotate_quant_bf16.cu", "rotate_quant_f32.cu", "rotate_quant_wide.cu", "rotate_quant_wide_f32.cu", "rotate_quant_a8_f16.cu",
           "rotate_quant_a8_bf16.cu", "rotate_quant_a8_f32.cu", "rotate_quant.cu", "rotate_quant_pass.cu", "a8_planes.cu", "block_rotate.cu", "gemm.cu", "gemm_tmem.cu", "gemm_fused.cu", "gemv.cu", "attention_prompt.cu", "attention_kv4.cu", "kv4_cache.cu", "api.cu", "api_attention.cu",
           "fp4_rows_f16.cu", "fp4_rows_bf16.cu", "fp4_rows_f32.cu", "norm_f16.cu", "norm_bf16.cu", "fp4_dequantize.cu", "fp4_gemm.cu", "fp4_token.cu", "api_fp4.cu",
           "pack.cpp"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: set NVCC or put the CUDA toolkit on PATH")


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [_nvcc(), *ARCH, *COMMON, "-c", os.path.join(CSRC, src), "-o", obj]
    if src.endswith(".cu"):
        cmd[1:1] = ["-Xptxas", "-v"] if verbose else []
    else:
        cmd += ["-Xcompiler", "-pthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compiling {src} failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    if verbose and (r.stdout or r.stderr):
        sys.stderr.write(r.stdout + r.stderr)
    return obj


def _stale(target: str) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    deps.append(__file__)
    return any(os.path.getmtime(d) > t for d in deps)


def _link(cmd: list[str], target: str) -> None:
    tmp = target + ".tmp"
    r = subprocess.run([tmp if word is None else word for word in cmd], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"linking {os.path.basename(target)} failed:\n{' '.join(map(str, cmd))}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, target)


def _build_calls() -> None:
    include = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(include, "Python.h")):
        sys.stderr.write(f"no Python.h in {include}: the calls of 4-bit floating point and of the norms are left out of the Python binding\n")
        return
    _link([os.environ.get("CC", "gcc"), "-O2", "-shared", "-fPIC", "-I", include, os.path.join(CSRC, "calls.c"), "-o", None, LIB,
           "-Wl,-rpath,$ORIGIN"], CALLS)
    untagged = os.path.join(PKG, "_calls.so")  # as it was named once: every interpreter would import it
    if os.path.exists(untagged):
        os.remove(untagged)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile and link what any source is newer than; return libqvla.so's path."""
    if force or _stale(LIB):
        os.makedirs(BUILD, exist_ok=True)
        with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
            objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
        _link([_nvcc(), *ARCH, "-shared", "-o", None, *objs, "-Xcompiler", "-pthread", "-Xlinker", "-soname=libqvla.so"], LIB)
    if force or _stale(CALLS):
        _build_calls()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
