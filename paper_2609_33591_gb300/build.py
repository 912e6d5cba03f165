"""Build libkint.so in-tree with nvcc for sm_103a (no torch extension machinery), and beside it
the Python module that marshals the serving calls (host code, g++, against torch's headers).

The translation units are compiled in parallel; the library is linked against the
shared CUDA runtime (the one PyTorch also loads), with an rpath to the CUDA
toolkit so it also loads on its own.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libkint.so")
EXT = os.path.join(BUILD, "_kint_serve.so")
EXT_SOURCE = os.path.join(CSRC, "serve_torch.cpp")
SOURCES = ["kint_api.cu", "kint_fwd.cu", "kint_bwd.cu", "kint_bwd_dkdv.cu", "kint_bwd_dkdv_rs.cu", "kint_bwd_fused.cu", "kint_probe.cu",
           "serve_api.cu", "serve_blocks.cu", "serve_rope.cu", "serve_cache.cu", "serve_attn_64.cu",
           "serve_attn_128.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libkint")
    return nvcc


def _cuda_lib_dir(nvcc: str) -> str:
    return os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "lib64")


def _inputs():
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)] + [__file__]
    return max(os.path.getmtime(p) for p in deps)


def _ext_command(out: str) -> list[str]:
    import torch
    home = os.path.dirname(torch.__file__)
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        raise RuntimeError("g++ not found: a C++ compiler is required to build the serving module")
    libs = os.path.join(home, "lib")
    return [cxx, "-O2", "-std=c++17", "-shared", "-fPIC", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-I", INCLUDE, "-I", sysconfig.get_paths()["include"], "-I", os.path.join(home, "include"),
            "-I", os.path.join(home, "include", "torch", "csrc", "api", "include"),
            "-I", os.path.join(os.path.dirname(_cuda_lib_dir(_nvcc())), "include"), EXT_SOURCE, "-o", out,
            "-L", libs, f"-Wl,-rpath,{libs}", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile (if stale) and return the path of libkint.so."""
    if not force and all(os.path.exists(f) and os.path.getmtime(f) >= _inputs() for f in (LIB, EXT)):
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    flags = ARCH + ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", INCLUDE]
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(BUILD, src.replace(".cu", f".{os.getpid()}.o"))
        objs.append(obj)
        cmd = [nvcc, *flags, "-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    ext_tmp = EXT + f".tmp{os.getpid()}"
    cmd = _ext_command(ext_tmp)
    procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = []
    for cmd, pr in procs:
        out, _ = pr.communicate()
        if pr.returncode != 0:
            failed.append(" ".join(cmd) + "\n" + out)
        elif verbose and out.strip():
            print(out, file=sys.stderr)
    if failed:
        for o in (*objs, ext_tmp):
            if os.path.exists(o):
                os.remove(o)
        raise RuntimeError("libkint build failed:\n" + "\n".join(failed))
    tmp = LIB + f".tmp{os.getpid()}"
    libdir = _cuda_lib_dir(nvcc)
    link = [nvcc, *ARCH, "-shared", "-cudart", "shared", "-o", tmp, *objs, "-Xlinker", f"-rpath={libdir}"]
    res = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    for o in objs:
        if os.path.exists(o):
            os.remove(o)
    if res.returncode != 0:
        os.remove(ext_tmp)
        raise RuntimeError("libkint link failed:\n" + " ".join(link) + "\n" + res.stdout)
    os.replace(tmp, LIB)
    os.replace(ext_tmp, EXT)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
