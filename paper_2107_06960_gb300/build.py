"""Build libmafat.so in-tree with nvcc for sm_103a.

Compiles each translation unit in parallel, then links one shared library
next to this file.  The library statically links the CUDA runtime and looks
up the driver's tensor-map encoder at run time, so it needs no libcuda at
link time and builds on a machine without a GPU.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmafat.so")
MATCH = os.path.join(HERE, "_match" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))  # the binding's, C for CPython
SOURCES = ["planner.cpp", "order.cpp", "runtime.cpp", "search.cpp", "kernel_fp32.cu", "kernel_tc.cu", "noalloc.cu",
           "attention.cpp", "attn_simt.cu", "attn_rows.cu", "attn_tc.cu", "attn_tc_tree.cu", "attn_join.cu", "rms_norm.cu",
           "decode.cpp", "block_norm.cu", "rotary.cu", "logits.cu"]
HEADERS = ["planner.h", "device_types.h", "kernels.h", "sched.cuh", "attention.h", "attn_common.cuh",
           "attn_tc.cuh", "decode.h", "lm_checks.h", "row_common.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc():
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    p = os.path.join(cuda, "bin", "nvcc")
    return p if os.path.exists(p) else (shutil.which("nvcc") or "nvcc")


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _compile(src, extra):
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    deps = [os.path.join(CSRC, src)] + [os.path.join(CSRC, h) for h in HEADERS] + \
           [os.path.join(ROOT, "include", "mafat.h"), __file__]
    if not _stale(obj, deps):
        return obj
    cmd = [_nvcc(), "-std=c++17", "-O3", "-lineinfo", "-Xcompiler", "-fPIC,-Wall",
           "-I", os.path.join(ROOT, "include")] + ARCH + extra + ["-c", os.path.join(CSRC, src), "-o", obj + ".tmp"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("nvcc failed for %s:\n%s%s" % (src, r.stdout, r.stderr))
    os.replace(obj + ".tmp", obj)
    return obj


def _build_match(force):
    src = os.path.join(CSRC, "match.c")
    if not force and not _stale(MATCH, [src, os.path.join(ROOT, "include", "mafat.h"), __file__]):
        return
    tmp = MATCH + ".tmp.%d" % os.getpid()
    cmd = ["gcc", "-O2", "-std=c11", "-Wall", "-fPIC", "-shared", "-I", sysconfig.get_paths()["include"], src, "-o", tmp]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
        why = r.stdout + r.stderr if r.returncode != 0 else None
    except OSError as e:
        why = str(e)
    if why is None:
        os.replace(tmp, MATCH)
        return
    # the binding does without it, and must not find one of other sources
    if os.path.exists(MATCH):
        os.remove(MATCH)
    warnings.warn("_match is not built, calls will take the host 2 us longer:\n%s" % why, RuntimeWarning)


def build(force: bool = False, extra=None) -> str:
    """Compile (if needed) and return the path of libmafat.so."""
    _build_match(force)
    extra = list(extra or [])
    os.makedirs(BUILD, exist_ok=True)
    if force:
        for f in os.listdir(BUILD):
            os.remove(os.path.join(BUILD, f))
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(lambda s: _compile(s, extra), SOURCES))
    if force or _stale(LIB, objs):
        tmp = LIB + ".tmp.%d" % os.getpid()
        cmd = [_nvcc(), "-shared"] + ARCH + objs + ["-o", tmp]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("link failed:\n%s%s" % (r.stdout, r.stderr))
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
