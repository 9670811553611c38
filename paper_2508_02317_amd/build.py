"""Build libmoe_gfx950.so (HIP, gfx950 only) in-tree with hipcc, and beside it _marshal.so, which carries torch tensors into it."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libmoe_gfx950.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
BUILD_DIR = os.path.join(ROOT, "_build")

SOURCES = ["api.hip", "route.hip", "permute.hip", "gemm_f32.hip", "gemm_bf16.hip", "rope.hip", "attn_decode.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 VALU forms (compiler flag for the device pass; the host pass ignores it)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build_library(verbose=False, extra_flags=()):
    """Compile every source and link the shared library; raises on any compiler error."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src):
        obj = os.path.join(BUILD_DIR, src.replace(".hip", ".o"))
        cmd = [hipcc, *HIPCC_FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj]
        res = subprocess.run(cmd, capture_output=True, text=True)
        log = "\n".join(l for l in (res.stdout + res.stderr).splitlines()
                        if "not a recognized feature for this target" not in l)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed on %s:\n%s" % (src, log))
        if verbose and log.strip():
            print(log, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stdout + res.stderr)
    build_marshal()
    return LIB


def build_marshal():
    """csrc/marshal.cpp as a Python extension module (host code only).  libmoe.py marshals through ctypes where it is missing: the same
    calls at some microseconds more each, so a host without Python's or torch's headers is told and not stopped."""
    import sysconfig
    if os.path.exists(MARSHAL):
        os.remove(MARSHAL)                             # never one of another build
    try:
        import torch
        troot = os.path.dirname(torch.__file__)
        abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    except (ImportError, AttributeError) as e:
        print("_marshal.so is not built: %s" % e, file=sys.stderr)
        return None
    inc, lib = os.path.join(troot, "include"), os.path.join(troot, "lib")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % abi, "-I", inc,
           "-I", os.path.join(inc, "torch", "csrc", "api", "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"),
           os.path.join(CSRC, "marshal.cpp"), "-o", MARSHAL, "-L", PKG, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN", "-L", lib, "-lc10", "-ltorch_cpu",
           "-ltorch_python"]
    try:
        res = subprocess.run(cmd, capture_output=True, text=True)
        log = res.stdout + res.stderr if res.returncode != 0 else ""
    except OSError as e:
        log = str(e)
    if log:
        print("_marshal.so is not built (calls are marshalled through ctypes):\n" + log[-2000:], file=sys.stderr)
        return None
    return MARSHAL


if __name__ == "__main__":
    print(build_library(verbose=True, extra_flags=tuple(sys.argv[1:])))
