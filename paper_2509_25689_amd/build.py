"""Build the HIP libraries for gfx950, in-tree.

Every source under ``csrc/`` is compiled with hipcc (one process per file, in
parallel) and linked into ``paper_2509_25689_amd/libmoeq.so``; ``peaks/`` (the
benchmark's measured roofline denominators) into ``libmoeq_peaks.so``; the
attention operators' binding to torch (host code, g++) into ``_attention.so``
beside them, unless torch, g++ or Python's headers are missing: the libraries
need hipcc alone.  Always recompiles: this is the "does it build" step."""
import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libmoeq.so")
BINDING = os.path.join(PKG, "binding", "attention.cpp")
BINDING_LIB = os.path.join(PKG, "_attention.so")
PEAKS = os.path.join(PKG, "peaks")
PEAKS_LIB = os.path.join(PKG, "libmoeq_peaks.so")
ARCH = "gfx950"

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    # never let the compiler form packed fp32 arithmetic
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def hipcc():
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def _compile(src):
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [hipcc(), *FLAGS, "-x", "hip", "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _link(objs, lib):
    tmp = lib + ".tmp"
    cmd = [hipcc(), "-shared", f"--offload-arch={ARCH}", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)


def _binding_lacks():
    """What this machine lacks to build the attention operators' binding, or None."""
    try:
        import torch
    except ImportError:
        return "torch"
    if not os.path.exists(os.path.join(os.path.dirname(torch.__file__), "include", "ATen", "ATen.h")):
        return "torch's headers"
    if not shutil.which("g++"):
        return "g++"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    return None


def _compile_binding():
    """The attention operators' binding to torch: host code only, so that a call
    costs the interpreter one step."""
    import torch
    tdir = os.path.join(os.path.dirname(torch.__file__), "include")
    obj = os.path.join(BUILD, "binding_attention.o")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-c", BINDING, "-o", obj,
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
           "-isystem", tdir, "-isystem", os.path.join(tdir, "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"]]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _link_binding(obj):
    import torch
    tlib = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = BINDING_LIB + ".tmp"
    cmd = ["g++", "-shared", obj, "-o", tmp, "-L", tlib, "-ltorch_python", "-ltorch", "-ltorch_cpu",
           "-lc10", "-L", PKG, "-l:libmoeq.so", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING_LIB)


def _sources(d):
    return sorted(os.path.join(d, f) for f in os.listdir(d) if f.endswith((".hip", ".cpp")))


def build(verbose=False):
    os.makedirs(BUILD, exist_ok=True)
    srcs = _sources(CSRC)
    psrcs = _sources(PEAKS)
    lacks = _binding_lacks()
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs) + len(psrcs) + 1)) as ex:
        binding = None if lacks else ex.submit(_compile_binding)
        objs = list(ex.map(_compile, srcs + psrcs))
    _link(objs[:len(srcs)], LIB)
    _link(objs[len(srcs):], PEAKS_LIB)
    if binding:
        _link_binding(binding.result())
    else:
        # one of an earlier build would not fit these sources
        if os.path.exists(BINDING_LIB):
            os.remove(BINDING_LIB)
        print(f"without {lacks}: {BINDING_LIB} (the attention operators' binding to torch) is not built")
    if verbose:
        print(f"built {LIB} and {PEAKS_LIB}" + (f" and {BINDING_LIB}" if binding else ""))
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
