"""Compile the HIP sources under csrc/ into libra.so next to this file (gfx950 only), and the host code of the binding into _calls.so where there
is a host compiler and the headers of Python and torch."""
import os
import shlex
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libra.so")
CALLS = os.path.join(HERE, "_calls.so")      # host code: short-cuts of binding.py (csrc/calls.cpp)
SOURCES = ["api.hip", "attend.hip", "search.hip", "decode.hip", "flat.hip", "knn.hip", "knn_order.hip", "knn_filter.hip", "project.hip",
           "quant.hip", "kv4.hip", "q4.hip", "paged.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]
# knn.hip: scores are compared as numbers (a NaN score, from non-finite inputs, never reaches a
# list either way); without this every fmaxf of the selection's max tree first canonicalises
# its inputs with an instruction of its own
EXTRA = {"knn.hip": ["-fno-honor-nans"]}


def _calls_command():
    """-> the command, and what is missing for it (None: nothing)."""
    try:
        import torch
    except ImportError:
        return [], "torch"
    at, python, cxx = os.path.dirname(torch.__file__), sysconfig.get_paths()["include"], shlex.split(os.environ.get("CXX") or "g++")
    headers = [os.path.join(python, "Python.h"), os.path.join(at, "include", "torch", "csrc", "autograd", "python_variable.h")]
    missing = [f for f in headers if not os.path.exists(f)] + ([] if shutil.which(cxx[0]) else [cxx[0]])
    return [*cxx, "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            "-I", os.path.join(ROOT, "include"), "-I", os.path.join(at, "include"), "-I", os.path.join(at, "include", "torch", "csrc", "api", "include"),
            "-I", python, os.path.join(CSRC, "calls.cpp"), "-o", CALLS,
            "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"], (", ".join(missing) or None)


def build(verbose=True):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    for s in SOURCES:
        o = os.path.join(CSRC, s.replace(".hip", ".o"))
        objs.append(o)
        cmd = [hipcc, *FLAGS, *EXTRA.get(s, []), "-c", os.path.join(CSRC, s), "-o", o]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    # (one of other sources would be taken for this one)
    if os.path.exists(CALLS):
        os.remove(CALLS)
    cmd, missing = _calls_command()
    if missing:
        print(f"_calls.so is not built, the calls around a cache in pages are checked in Python: {missing} is missing", flush=True)
    else:
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append(("calls.cpp", subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for s, p in procs:
        out = p.communicate()[0].decode()
        noise = "is not a recognized feature for this target"
        out = "\n".join(l for l in out.splitlines() if noise not in l)
        if out.strip() and verbose:
            print(out)
        if p.returncode:
            failed.append((s, f"the compiler failed on {s}:\n{out}"))
    if any(s != "calls.cpp" for s, _ in failed):
        raise RuntimeError("\n".join(said for _, said in failed))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    if failed:                      # (the library does without)
        raise RuntimeError(failed[0][1])
    return LIB


if __name__ == "__main__":
    build()
    print("built", LIB)
