"""Builds liblrqat.so in-tree for sm_103a (nvcc, one -gencode, parallel compiles), and the Python binding's short way into
it (g++, against the installed torch; without torch or Python's headers, or where it does not compile, the binding does
without).

Usage: python -m paper_2406_06385_gb300.build [--force]
"""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(PKG, "_build")
LIB_DIR = os.path.join(PKG, "_lib")
LIB_PATH = os.path.join(LIB_DIR, "liblrqat.so")

SOURCES = ["elementwise.cu", "fused_gemm.cu", "fused_pair.cu", "dw.cu", "dw_pair.cu", "merge.cu", "optim.cu", "norm.cu",
           "rope.cu", "kv_blocks.cu", "kv_cache.cu", "kv_attn.cu", "kv_prompt.cu", "lrqat_api.cu"]
HEADERS = ["kernels.h", "merge.h", "ptx.cuh", "quant.cuh", "serve.h", "serve.cuh",
           "attn.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]


def binding_path() -> str:
    """Where the binding's short way for the installed torch lies, "" without a torch for CUDA or Python's headers."""
    spec = importlib.util.find_spec("torch")
    if (not spec or not os.path.exists(os.path.join(os.path.dirname(spec.origin), "lib", "libc10_cuda.so"))
            or not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))):
        return ""
    return os.path.join(LIB_DIR, f"lrqat_binding-{importlib.metadata.version('torch').split('+')[0]}-{sys.implementation.cache_tag}.so")


def binding_command(target: str):
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    include = [sysconfig.get_paths()["include"], os.path.join(torch, "include"), cuda, INCLUDE]
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-w"] + [f"-I{i}" for i in include]
            + [os.path.join(CSRC, "binding.cpp"), "-o", target, f"-L{LIB_DIR}", "-l:liblrqat.so", "-Wl,-rpath,$ORIGIN",
               f"-L{os.path.join(torch, 'lib')}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])


def nvcc() -> str:
    cand = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build liblrqat")
    return cand


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every CUDA source and link liblrqat.so; returns its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    os.makedirs(LIB_DIR, exist_ok=True)
    cc = nvcc()
    headers = [os.path.join(CSRC, h) for h in HEADERS] + [os.path.join(INCLUDE, "lrqat.h")]
    objs = []
    jobs = []
    for src in SOURCES:
        path = os.path.join(CSRC, src)
        obj = os.path.join(BUILD_DIR, src.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, [path] + headers):
            jobs.append([cc] + NVCC_FLAGS + ["-c", path, "-o", obj])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    with ThreadPoolExecutor(max_workers=len(jobs) or 1) as ex:
        for cmd, r in ex.map(run, jobs):
            if verbose or r.returncode != 0:
                sys.stderr.write(r.stdout + r.stderr)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed: {' '.join(cmd)}")
    if force or jobs or _stale(LIB_PATH, objs):
        tmp = LIB_PATH + ".tmp"
        cmd = [cc] + ARCH + ["-shared", "-Xcompiler", "-fPIC", "-o", tmp] + objs
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError("linking liblrqat.so failed")
        os.replace(tmp, LIB_PATH)
    binding = binding_path()
    source = [os.path.join(CSRC, "binding.cpp"), os.path.join(INCLUDE, "lrqat.h")]
    if binding and (force or _stale(binding, source)):
        try:
            r = subprocess.run(binding_command(binding + ".tmp"), capture_output=True, text=True)
            failed = r.stdout + r.stderr if r.returncode else None
        except OSError as e:
            failed = str(e)
        if failed is None:
            os.replace(binding + ".tmp", binding)
        else:
            sys.stderr.write(f"{failed}\ncompiling the binding's short way failed; the binding does without\n")
            if os.path.exists(binding):      # of older sources than the library
                os.remove(binding)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
