"""Builds libasap_moe.so in-tree with nvcc for sm_103a (GB300).

    python -m paper_2606_22541_gb300.build [--force] [--verbose]

The translation units compile in parallel; the library links the CUDA
runtime statically and resolves the one driver entry point it needs
(cuTensorMapEncodeTiled) at run time, so it loads on machines without a GPU.
"""
import contextlib
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
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libasap_moe.so")
SOURCES = ["api.cu", "gemm_tc.cu", "gemm_pair.cu", "gemm_fp8.cu", "route.cu", "route_tc.cu", "permute.cu", "mailbox.cu",
           "few.cu", "fp8_ops.cu"]
HEADERS = [os.path.join(CSRC, "common.cuh"), os.path.join(CSRC, "internal.h"), os.path.join(CSRC, "gemm_sched.cuh"), os.path.join(CSRC, "gemm_config.h"),
           os.path.join(CSRC, "pair.cuh"), os.path.join(CSRC, "few.h"), os.path.join(CSRC, "e4m3.cuh"),
           os.path.join(INCLUDE, "asap_moe.h")]
MARSHAL = os.path.join(PKG, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))  # loaded by this Python version only
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-fvisibility=hidden",
         "-I", INCLUDE, "-I", CSRC]


def _nvcc():
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if c and (os.path.sep not in c or os.path.exists(c)):
            return c
    return "nvcc"


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force=False, verbose=False, extra_flags=()):
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    objs, jobs = [], []
    for s in SOURCES:
        src = os.path.join(CSRC, s)
        obj = os.path.join(BUILD, s.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, [src] + HEADERS):
            jobs.append([nvcc, *ARCH, *FLAGS, *extra_flags, "-c", src, "-o", obj])

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        return cmd, r

    with ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 4))) as ex:
        for cmd, r in ex.map(run, jobs):
            if verbose and r.stderr:
                print(r.stderr, file=sys.stderr)
            if r.returncode != 0:
                raise RuntimeError("nvcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + ".tmp"
        cmd = [nvcc, *ARCH, "-shared", "-Xcompiler", "-fPIC,-fvisibility=hidden", "-o", tmp, *objs]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("link failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
        os.replace(tmp, LIB)
    build_marshal(force)
    return LIB


def build_marshal(force=False):
    """The Python binding's marshalling of the short calls, where Python's
    headers and a C compiler are installed (without it they are marshalled in
    Python)."""
    src, include = os.path.join(CSRC, "marshal.c"), sysconfig.get_paths()["include"]
    untagged = os.path.join(PKG, "_marshal.so")  # any Python version would load it
    with contextlib.suppress(FileNotFoundError):
        os.remove(untagged)
    gcc = shutil.which("gcc")
    if gcc is None or not os.path.exists(os.path.join(include, "Python.h")) or not (force or _stale(MARSHAL, [src])):
        return
    tmp = MARSHAL + ".tmp"
    cmd = [gcc, "-O2", "-Wall", "-shared", "-fPIC", "-fvisibility=hidden", "-I", include, src, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("gcc failed:\n" + " ".join(cmd) + "\n" + r.stdout + r.stderr)
    os.replace(tmp, MARSHAL)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
