"""Build libw8a8.so in-tree with nvcc for sm_103a (GB300).

Each ``csrc/*.cu`` compiles to an object under ``_build/`` (in parallel), and the objects link
into ``paper_2608_28003_gb300/libw8a8.so``; ``csrc/calls.cc``, the binding's marshalling, compiles
to the extension module ``_calls.so`` beside it.  A source newer than its object, or a header newer
than the library, triggers a rebuild; ``_calls.so`` reads tensors where PyTorch's headers say they lie, so another PyTorch or
interpreter than it was compiled for, or another command, does too.  No fast-math: every rounding the header documents is an
IEEE operation.
"""
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
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libw8a8.so")
CALLS = os.path.join(PKG, "_calls.so")
CALLS_STAMP = os.path.join(BUILD, "calls.stamp")  # what _calls.so was compiled with

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
              "-Xptxas", "-warn-spills"]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libw8a8")


def _headers():
    return glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _compile(src: str, obj: str, verbose: bool) -> None:
    cmd = [nvcc(), *ARCH, *NVCC_FLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed for {os.path.basename(src)}:\n{r.stdout}\n{r.stderr}")
    if verbose and (r.stdout.strip() or r.stderr.strip()):
        print(r.stdout, r.stderr)


def torch_id() -> str:
    """The PyTorch that _calls.so is compiled for, which it compares with the one it is loaded beside."""
    import torch
    return f"{torch.__version__} {torch.version.git_version}"


def _calls_flags() -> list:
    import torch  # for its headers and libraries: the module reads tensors through them
    at = os.path.dirname(torch.__file__)
    return ["-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DW8A8_TORCH="{torch_id()}"',
            "-I", sysconfig.get_paths()["include"], "-isystem", os.path.join(at, "include"),
            "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
            "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"]


def _calls_stamp() -> str:
    """What _calls.so depends on beside its sources."""
    return "\n".join([*_calls_flags(), sysconfig.get_config_var("SOABI") or "", sys.version])


def _compile_calls(src: str) -> None:
    cxx = shutil.which(os.environ.get("CXX", "g++")) or shutil.which("c++")
    if cxx is None:
        raise RuntimeError("g++ not found: it compiles the binding's calls")
    tmp = CALLS + ".tmp"
    flags = _calls_flags()
    libs = flags.index("-L")
    r = subprocess.run([cxx, *flags[:libs], src, "-o", tmp, *flags[libs:]], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for {os.path.basename(src)}:\n{r.stdout}\n{r.stderr}")
    if os.path.exists(CALLS_STAMP):  # a module never lies beside another one's stamp
        os.remove(CALLS_STAMP)
    os.replace(tmp, CALLS)
    with open(CALLS_STAMP, "w") as f:
        f.write(_calls_stamp())


def _calls_stale(newest: float) -> bool:
    if not os.path.exists(CALLS) or os.path.getmtime(CALLS) < newest or not os.path.exists(CALLS_STAMP):
        return True
    with open(CALLS_STAMP) as f:
        return f.read() != _calls_stamp()


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every CUDA source for sm_103a and link libw8a8.so, and compile the binding's calls.
    Returns the library path."""
    os.makedirs(BUILD, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    hdr_mtime = max([os.path.getmtime(h) for h in _headers()] + [0.0])
    jobs = []
    for s in srcs:
        o = os.path.join(BUILD, os.path.basename(s)[:-3] + ".o")
        stale = force or not os.path.exists(o) or os.path.getmtime(o) < max(os.path.getmtime(s), hdr_mtime)
        jobs.append((s, o, stale))
    with cf.ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 4))) as ex:
        futs = [ex.submit(_compile, s, o, verbose) for s, o, stale in jobs if stale]
        calls = os.path.join(CSRC, "calls.cc")
        if force or _calls_stale(max(os.path.getmtime(calls), hdr_mtime)):
            futs.append(ex.submit(_compile_calls, calls))
        for f in futs:
            f.result()
    objs = [o for _, o, _ in jobs]
    newest = max(os.path.getmtime(o) for o in objs)
    if force or not os.path.exists(LIB) or os.path.getmtime(LIB) < newest:
        tmp = LIB + ".tmp"
        cmd = [nvcc(), *ARCH, "-shared", "-o", tmp, *objs, "-cudart", "static"]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link of libw8a8.so failed:\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
