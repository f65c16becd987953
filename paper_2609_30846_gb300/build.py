"""Builds the GPU library ``libipmhsa.so`` in-tree with nvcc for sm_103a.

The library is the whole product path: the C ABI of include/ip_mhsa.h and
the CUDA kernels behind it.  Beside it, where torch is installed, the host compiler
builds ``ip_torch.so``, the native short forms of some Python calls.  Nothing here needs a
GPU; nvcc cross-compiles.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libipmhsa.so")
SOURCES = [os.path.join(CSRC, f) for f in ("ip_mhsa.cu", "ip_linear.cu", "ip_norm.cu",
                                           "ip_block.cu", "ip_scaled.cu", "ip_kv4.cu")]
DEPS = SOURCES + [os.path.join(CSRC, f) for f in ("ip_mhsa_kernels.cuh", "ip_linear_kernels.cuh",
                                                  "ip_norm_kernels.cuh", "ip_block_kernels.cuh",
                                                  "ip_scaled_kernels.cuh", "ip_kv4_kernels.cuh", "ip_real.cuh",
                                                  "ip_ptx.cuh",
                                                  "ip_probe.cuh", "ip_host_util.h")] + [
    os.path.join(INCLUDE, "ip_mhsa.h")]
TORCH_LIB = os.path.join(PKG, "ip_torch.so")
TORCH_SOURCE = os.path.join(CSRC, "ip_torch.cpp")
ARCH = "-gencode=arch=compute_103a,code=sm_103a"


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the GPU library cannot be built")


FLAGS = [ARCH, "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC"]


def compile_command(src: str, obj: str) -> list[str]:
    return [nvcc()] + FLAGS + ["-I" + INCLUDE, "-c", "-o", obj, src]


def link_command(objs: list[str], out: str) -> list[str]:
    return [nvcc(), ARCH, "-shared", "-o", out] + objs


def _torch_dir():
    """Folder of a torch built with CUDA, None without one."""
    spec = importlib.util.find_spec("torch")
    path = os.path.dirname(spec.origin) if spec is not None and spec.origin else None
    return path if path and os.path.exists(os.path.join(path, "lib", "libc10_cuda.so")) else None


def torch_command(out: str) -> list[str]:
    torch = _torch_dir()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    dirs = [INCLUDE, os.path.join(torch, "include"), os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    libs = os.path.join(torch, "lib")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-o", out, TORCH_SOURCE] + [
        "-I" + d for d in dirs] + ["-L" + libs, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def torch_extension():
    """Path of ip_torch.so, None without a torch for it."""
    return TORCH_LIB if _torch_dir() is not None else None


def _fresh(lib: str, deps: list[str]) -> bool:
    if not os.path.exists(lib):
        return False
    t = os.path.getmtime(lib)
    return all(os.path.getmtime(d) <= t for d in deps)


def up_to_date() -> bool:
    return _fresh(LIB, DEPS) and (_torch_dir() is None or
                                  _fresh(TORCH_LIB, [TORCH_SOURCE, os.path.join(INCLUDE, "ip_mhsa.h")]))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile (if stale) both libraries and return the path of libipmhsa.so."""
    if not force and up_to_date():
        return LIB
    tag = f".tmp{os.getpid()}"
    objs = [os.path.join(CSRC, os.path.basename(s) + tag + ".o") for s in SOURCES]
    tmp_torch = TORCH_LIB + tag
    cmds = [compile_command(src, obj) for src, obj in zip(SOURCES, objs)]
    if _torch_dir() is not None:
        cmds.append(torch_command(tmp_torch))
    try:
        # the translation units compile in parallel, then one link
        procs = []
        for cmd in cmds:
            if verbose:
                print(" ".join(cmd), flush=True)
            procs.append((cmd, subprocess.Popen(cmd, cwd=CSRC)))
        for cmd, p in procs:
            if p.wait() != 0:
                raise subprocess.CalledProcessError(p.returncode, cmd)
        tmp = LIB + tag
        subprocess.run(link_command(objs, tmp), check=True, cwd=CSRC)
        os.replace(tmp, LIB)
        if os.path.exists(tmp_torch):
            os.replace(tmp_torch, TORCH_LIB)
    finally:
        for obj in objs + [tmp_torch]:
            if os.path.exists(obj):
                os.unlink(obj)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
