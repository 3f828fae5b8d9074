"""Build libpsppo.so (nvcc, sm_103a only) and the module of small calls (the host compiler) in place.

Each translation unit compiles in parallel; the objects link into
paper_2606_29758_gb300/libpsppo.so with the CUDA runtime linked statically, so the
library needs only the driver at run time. The other is a Python module over torch's headers
that makes the block operators' small calls; nothing in libpsppo.so depends on it, and where it
cannot be built (no torch, no compiler) the calls go through ctypes. Its file's name says which
torch and which Python it was compiled for.
No cmake, no torch extension machinery.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libpsppo.so")
CALLS_SOURCE = "small_calls.cpp"
SOURCES = ["psppo_api.cu", "lmhead_bf16.cu", "lmhead_f32.cu", "fwd_static_scratch.cu", "design.cu", "ffn.cu", "block_ops.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _compile(src: str, verbose_ptxas: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [nvcc(), *ARCH, "-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-O2", "-I", INCLUDE, "-I", CSRC,
           "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose_ptxas:
        cmd.insert(1, "-Xptxas=-v")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    if verbose_ptxas:
        sys.stderr.write(r.stderr)
    return obj


def calls_path() -> str:
    """The module of small calls for the running torch and Python."""
    import torch
    return os.path.join(PKG, f"_calls-{torch.__version__}-{(torch.version.git_version or '')[:12]}-"
                             f"{sysconfig.get_config_var('SOABI')}.so")


def _build_calls() -> None:
    import torch
    out = calls_path()
    base = os.path.dirname(torch.__file__)
    dirs = [INCLUDE, os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"),
            sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(nvcc())), "include")]
    tmp = out + f".tmp{os.getpid()}"
    cmd = [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *(f"-I{d}" for d in dirs),
           os.path.join(CSRC, CALLS_SOURCE), "-o", tmp, "-L" + os.path.join(base, "lib"),
           "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed for {CALLS_SOURCE}:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, out)


def _remove_calls() -> None:
    try:
        os.remove(calls_path())
    except (ImportError, FileNotFoundError):
        pass


def _older(out: str, sources) -> bool:
    if not os.path.exists(out):
        return True
    deps = [*sources, *(os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)), os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > os.path.getmtime(out) for p in deps)


def _lib_stale() -> bool:
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != CALLS_SOURCE])


def _calls_stale() -> bool:
    try:
        out = calls_path()
    except ImportError:   # (no torch: nothing would use it)
        return False
    return _older(out, [os.path.join(CSRC, CALLS_SOURCE)])


def _stale() -> bool:
    return _lib_stale() or _calls_stale()


def build(force: bool = False, verbose_ptxas: bool = False) -> str:
    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        calls = ex.submit(_build_calls) if force or _calls_stale() else None
        if force or _lib_stale():
            _build_lib(ex, verbose_ptxas)
        if calls is not None:
            try:
                calls.result()
            except Exception as e:   # (the library is complete without it; an older one may not fit it)
                _remove_calls()
                warnings.warn(f"the module of small calls is not built, the block operators' calls go through ctypes: {e}")
    return LIB


def _build_lib(ex: ThreadPoolExecutor, verbose_ptxas: bool) -> None:
    os.makedirs(BUILD, exist_ok=True)
    objs = list(ex.map(lambda s: _compile(s, verbose_ptxas), SOURCES))
    tmp = LIB + f".tmp{os.getpid()}"
    r = subprocess.run([nvcc(), *ARCH, "-shared", "-o", tmp, *objs], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose_ptxas="-v" in sys.argv))
