"""Builds libfsx.so (the C-ABI CUDA library) in-tree for sm_103a.

Each .cu translation unit is compiled in parallel with nvcc, then linked into
``paper_2607_15621_gb300/_lib/libfsx.so`` with the CUDA runtime linked
statically, so the library loads on machines without a GPU. ``_lib/_calls.so``
is the Python extension that passes torch tensors to some of its entry points.

    python -m paper_2607_15621_gb300.build
"""
from __future__ import annotations

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
OUT_DIR = os.path.join(PKG, "_lib")
BUILD_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(OUT_DIR, "libfsx.so")
CALLS = os.path.join(OUT_DIR, "_calls.so")
SOURCES = ["fsx.cu", "launch.cu", "gemm_tc.cu", "gemm_stream.cu", "gemm_res.cu", "attention.cu", "attention_tc.cu", "embed_head.cu",
           "attention_noalloc.cu", "tick_persistent.cu", "append.cu", "paper_tokens.cu", "session.cu",
           "llm.cu", "cache8.cu", "prompt_attention.cu", "tree_attention.cu", "tree_tc.cu", "pages.cu",
           "rotary.cu", "paged_attention.cu", "page_select.cu", "page_table.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-pthread",
         "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include")]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("command failed:\n" + " ".join(cmd) + "\n" + res.stdout + res.stderr)
    return res.stdout + res.stderr


def _torch() -> str:
    """Where torch lies; empty: nowhere. It is not imported."""
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec is not None and spec.origin else ""


def calls_lacks() -> str:
    """What a build of the extension module lacks on this machine; empty: nothing."""
    at, python, cxx = _torch(), os.path.join(sysconfig.get_paths()["include"], "Python.h"), os.environ.get("CXX", "g++")
    header = os.path.join(at, "include", "torch", "csrc", "autograd", "python_variable.h")
    lacks = ["torch" if not at else "" if os.path.exists(header) else header,
             "" if os.path.exists(python) else python, "" if shutil.which(cxx) else cxx]
    return ", ".join(x for x in lacks if x)


def _build_calls() -> str:
    """The extension module: plain C++ against this interpreter's and this torch's headers. Where they are missing it is left out:
    the library has no use for them."""
    lacks = calls_lacks()
    if os.path.exists(CALLS):
        os.remove(CALLS)  # of an earlier build
    if lacks:
        print(f"{CALLS} is not built: no {lacks}", file=sys.stderr)
        return ""
    at = _torch()
    include = [sysconfig.get_paths()["include"], os.path.join(at, "include"),
               os.path.join(at, "include", "torch", "csrc", "api", "include"), os.path.join(ROOT, "include")]
    out = _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", *(x for i in include for x in ("-I", i)),
                os.path.join(CSRC, "calls.cpp"), "-o", CALLS + ".tmp", "-L" + os.path.join(at, "lib"), "-ltorch_python",
                "-ltorch_cpu", "-ltorch", "-lc10", "-ldl"])
    os.replace(CALLS + ".tmp", CALLS)
    return out


def build(verbose: bool = False, extra_flags=()) -> str:
    os.makedirs(OUT_DIR, exist_ok=True)
    os.makedirs(BUILD_DIR, exist_ok=True)
    cc = nvcc()
    objs = []
    cmds = []
    for src in SOURCES:
        obj = os.path.join(BUILD_DIR, src.replace(".cu", ".o"))
        objs.append(obj)
        cmds.append([cc, *ARCH, *FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj])
    with ThreadPoolExecutor(max_workers=len(cmds) + 1) as ex:
        calls = ex.submit(_build_calls)
        logs = list(ex.map(_run, cmds))
        tmp = LIB + ".tmp"
        logs.append(_run([cc, *ARCH, "-shared", "-Xcompiler", "-pthread", "-o", tmp, *objs]))
        os.replace(tmp, LIB)
        logs.append(calls.result())
    if verbose:
        print("".join(logs))
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv,
          extra_flags=("-Xptxas", "-v") if "--ptxas" in sys.argv else ())
    print(LIB)
