"""Builds csrc/*.cu into csrc/libefcp.so with nvcc for sm_100a, and csrc/efcp_marshal.cpp into
_marshal.so against the installed torch (both in-tree, no JIT cache)."""
import glob
import os
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(CSRC, "libefcp.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
MARSHAL_SRC = os.path.join(CSRC, "efcp_marshal.cpp")


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(
        os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(INCLUDE, "*.h"))


def _stale(target, deps):
    return not os.path.exists(target) or os.path.getmtime(target) < max(map(os.path.getmtime, deps))


def _bound_to() -> str:
    """What a build of _marshal.so fits: torch's C++ interface and the interpreter's."""
    import torch
    return f"torch {torch.__version__}, Python {sys.version_info.major}.{sys.version_info.minor}"


def _built_for() -> str:
    try:
        with open(MARSHAL + ".built_for") as f:
            return f.read()
    except OSError:
        return ""


def build_marshal(force: bool = False) -> str:
    """Compile _marshal.so when it is missing, older than its sources or built for another torch;
    return its path."""
    deps = [MARSHAL_SRC] + glob.glob(os.path.join(INCLUDE, "*.h"))
    if not force and not _stale(MARSHAL, deps) and _built_for() == _bound_to():
        return MARSHAL
    import torch
    root = os.path.dirname(torch.__file__)
    lib = os.path.join(root, "lib")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
           "-I", sysconfig.get_paths()["include"], "-I", os.path.join(root, "include"),
           "-I", os.path.join(root, "include", "torch", "csrc", "api", "include"), "-I", INCLUDE,
           "-I", os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"),
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-o", MARSHAL + ".tmp", MARSHAL_SRC,
           "-L", lib, "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda",
           "-L", CSRC, "-l:libefcp.so",
           f"-Wl,-rpath,{lib}", "-Wl,-rpath,$ORIGIN/csrc"]
    subprocess.run(cmd, check=True)
    os.replace(MARSHAL + ".tmp", MARSHAL)
    with open(MARSHAL + ".built_for", "w") as f:
        f.write(_bound_to())
    return MARSHAL


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile what is missing or older than its sources; return the CUDA library's path."""
    if force or _stale(LIB, _deps()):
        nvcc = os.environ.get("NVCC", "nvcc")
        flags = os.environ.get("EFCP_NVCC_FLAGS", "").split() + [  # e.g. -DEFCP_DEPTH=8
            "-std=c++17", "-O3", "-lineinfo", "-gencode", "arch=compute_100a,code=sm_100a",
            "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]
        if verbose:
            flags = ["-Xptxas", "-v"] + flags
        # the sources at the same time: the templates of one take as long as all the rest
        with tempfile.TemporaryDirectory() as tmp:
            objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in _sources()]
            jobs = [subprocess.Popen([nvcc] + flags + ["-c", "-o", o, s])
                    for s, o in zip(_sources(), objects)]
            failed = [s for s, j in zip(_sources(), jobs) if j.wait() != 0]
            if failed:
                raise RuntimeError("nvcc failed for " + ", ".join(failed))
            subprocess.run([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a",
                            "-o", LIB + ".tmp"] + objects, check=True)
        os.replace(LIB + ".tmp", LIB)
    build_marshal(force)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
