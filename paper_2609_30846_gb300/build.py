"""Builds the GPU library ``libipmhsa.so`` in-tree with nvcc for sm_103a.

The library is the whole product path: the C ABI of include/ip_mhsa.h and
the CUDA kernels behind it.  Beside it, where torch is installed, the host compiler
builds ``ip_torch.<python>-torch<version>.so``, the native short forms of some Python calls; the
library does not depend on it, and where it cannot be built (no Python headers, say) these
calls take their general forms.  Nothing here needs a GPU; nvcc cross-compiles.
"""
from __future__ import annotations

import importlib.util
import os
import re
import shutil
import subprocess
import sysconfig
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libipmhsa.so")
SOURCES = [os.path.join(CSRC, f) for f in ("ip_mhsa.cu", "ip_linear.cu", "ip_norm.cu",
                                           "ip_block.cu", "ip_scaled.cu", "ip_kv4.cu",
                                           "ip_rows.cu", "ip_fp4.cu", "ip_logprobs.cu")]
DEPS = SOURCES + [os.path.join(CSRC, f) for f in ("ip_mhsa_kernels.cuh", "ip_linear_kernels.cuh",
                                                  "ip_norm_kernels.cuh", "ip_block_kernels.cuh",
                                                  "ip_scaled_kernels.cuh", "ip_kv4_kernels.cuh", "ip_real.cuh",
                                                  "ip_rows_kernels.cuh", "ip_fp4_kernels.cuh", "ip_logprobs_kernels.cuh",
                                                  "ip_ptx.cuh",
                                                  "ip_probe.cuh", "ip_host_util.h")] + [
    os.path.join(INCLUDE, "ip_mhsa.h")]
TORCH_SOURCE = os.path.join(CSRC, "ip_torch.cpp")
TORCH_DEPS = [TORCH_SOURCE, os.path.join(INCLUDE, "ip_mhsa.h")]
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


def _torch_version() -> str:
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        return re.search(r"^__version__ = ['\"]([^'\"]+)['\"]", f.read(), re.M).group(1)


def torch_extension():
    """Path of the native short forms, None without a torch for them.  Its name holds the Python
    and the torch that it is built for: one of other versions is never loaded."""
    if _torch_dir() is None:
        return None
    return os.path.join(PKG, f"ip_torch.{sysconfig.get_config_var('SOABI')}-torch{_torch_version()}.so")


def _fresh(lib: str, deps: list[str]) -> bool:
    if not os.path.exists(lib):
        return False
    t = os.path.getmtime(lib)
    return all(os.path.getmtime(d) <= t for d in deps)


def _stale_extension(force: bool = False):
    """Path of the native short forms if they have to be built, else None."""
    try:
        ext = torch_extension()
    except Exception as exc:  # noqa: BLE001 - a torch that is not as expected
        _without_extension(exc)
        return None
    return ext if ext is not None and (force or not _fresh(ext, TORCH_DEPS)) else None


def _without_extension(why) -> None:
    warnings.warn(f"the native short forms cannot be built: {why}; the calls take their general forms",
                  RuntimeWarning, stacklevel=3)


def up_to_date() -> bool:
    return _fresh(LIB, DEPS) and _stale_extension() is None


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile (if stale) the library and the short forms and return the path of libipmhsa.so."""
    sources = SOURCES if force or not _fresh(LIB, DEPS) else []
    ext = _stale_extension(force)
    tag = f".tmp{os.getpid()}"
    objs = [os.path.join(CSRC, os.path.basename(s) + tag + ".o") for s in sources]
    tmp_ext = ext + tag if ext is not None else None

    def start(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        return cmd, subprocess.Popen(cmd, cwd=CSRC)

    try:
        # the translation units compile in parallel, then one link
        procs = [start(compile_command(src, obj)) for src, obj in zip(sources, objs)]
        ext_proc = None
        if ext is not None:
            try:
                ext_proc = start(torch_command(tmp_ext))[1]
            except Exception as exc:  # noqa: BLE001 - no compiler, say
                _without_extension(exc)
        for cmd, p in procs:
            if p.wait() != 0:
                raise subprocess.CalledProcessError(p.returncode, cmd)
        if sources:
            tmp = LIB + tag
            subprocess.run(link_command(objs, tmp), check=True, cwd=CSRC)
            os.replace(tmp, LIB)
        if ext_proc is not None:
            if ext_proc.wait() == 0:
                os.replace(tmp_ext, ext)
            else:
                _without_extension(f"the compiler returned {ext_proc.returncode}")
    finally:
        for path in objs + ([tmp_ext] if tmp_ext is not None else []):
            if os.path.exists(path):
                os.unlink(path)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
