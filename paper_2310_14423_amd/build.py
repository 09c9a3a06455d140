"""Builds libqsr.so (the C-ABI library) for gfx950 with hipcc, and the Python extension that calls it with torch tensors, in-tree."""
import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(os.path.dirname(PKG), "include")
LIB = os.path.join(PKG, "libqsr.so")
CALLS = os.path.join(PKG, "_calls.so")

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",   # no packed-fp32 instructions
         # a kernel's first arguments in its registers when a wavefront starts, without a load: 1 to 1.5 % of the chains of short
         # launches (two encoder blocks of 1040 tokens 184.8 -> 181.7 us); single iterations of least squares take the same time
         "-mllvm", "-amdgpu-kernarg-preload-count=16",
         "-Wall", "-Wno-unused-function"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def build(verbose=False):
    cmd = ["hipcc"] + FLAGS + ["-I", INCLUDE, "-I", CSRC] + sources() + ["-o", LIB + ".tmp"]
    if verbose:
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    os.replace(LIB + ".tmp", LIB)
    build_calls(verbose)
    return LIB


def headers():
    """The folders of the headers of torch and Python, and that of torch's libraries; None where headers are missing."""
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.origin:
        return None
    root, python = os.path.dirname(spec.origin), sysconfig.get_paths()["include"]
    found = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), python]
    needed = [os.path.join(found[0], "torch", "csrc", "autograd", "python_variable.h"), os.path.join(python, "Python.h")]
    return (found, os.path.join(root, "lib")) if all(os.path.exists(f) for f in needed) else None


def build_calls(verbose=False):
    """The extension behind operators.py: host code, against torch's headers and libqsr.so.  Where there are none the library is all
    that is built, and the operators' Python side raises when it is called."""
    got = headers()
    if got is None:
        print("no headers of torch and Python: %s is not built, and the operators can be called through the C ABI alone" % CALLS, file=sys.stderr)
        if os.path.exists(CALLS):       # one for another library would be worse than none
            os.remove(CALLS)
        return None
    import torch
    include, libs = got
    cmd = ["hipcc", "-no-hip-rt", "-x", "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(),
           "-I", INCLUDE] + [a for f in include for a in ("-isystem", f)] + [os.path.join(CSRC, "torch_calls.cpp"), "-o", CALLS + ".tmp",
           "-L", PKG, "-lqsr", "-L", libs, "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    os.replace(CALLS + ".tmp", CALLS)
    return CALLS


if __name__ == "__main__":
    print(build(verbose=True))
