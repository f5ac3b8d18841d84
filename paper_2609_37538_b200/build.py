"""Compiles csrc/*.cu into libavsg.so with nvcc for sm_100a, and the binding's extension modules with g++ (all in-tree)."""
import glob
import os
import subprocess
import sysconfig
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(_HERE), "include")
LIB = os.path.join(_HERE, "libavsg.so")
CALLS_SOURCE = os.path.join(CSRC, "python_calls.cpp")
CALLS = os.path.join(_HERE, "_python_calls" + sysconfig.get_config_var("EXT_SUFFIX"))      # (of this Python)
TENSOR_CALLS_SOURCE = os.path.join(CSRC, "tensor_calls.cpp")
TENSOR_CALLS = os.path.join(_HERE, "_tensor_calls" + sysconfig.get_config_var("EXT_SUFFIX"))      # (of this Python and this torch)

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-shared", "--use_fast_math",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale(srcs) -> bool:
    if not os.path.exists(LIB):
        return True
    deps = srcs + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    return any(os.path.getmtime(d) > os.path.getmtime(LIB) for d in deps)


def build_calls(force: bool = False):
    """The extension module that makes the binding's hot calls, rebuilt when a source is newer."""
    deps = [CALLS_SOURCE] + glob.glob(os.path.join(INCLUDE, "*.h"))
    if force or not os.path.exists(CALLS) or any(os.path.getmtime(d) > os.path.getmtime(CALLS) for d in deps):
        tmp = CALLS + ".tmp.%d" % os.getpid()
        subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-Wall", "-Wextra", "-Wno-missing-field-initializers",
                               "-fPIC", "-shared", "-fvisibility=hidden", "-I", sysconfig.get_paths()["include"], "-I", INCLUDE,
                               "-o", tmp, CALLS_SOURCE])
        os.replace(tmp, CALLS)
    return CALLS


def build_tensor_calls(force: bool = False):
    """The extension module that makes the calls with torch's tensors, rebuilt when a source is newer."""
    deps = [TENSOR_CALLS_SOURCE] + glob.glob(os.path.join(INCLUDE, "*.h"))
    if force or not os.path.exists(TENSOR_CALLS) or any(os.path.getmtime(d) > os.path.getmtime(TENSOR_CALLS) for d in deps):
        import torch
        root = os.path.dirname(torch.__file__)
        headers = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), "/usr/local/cuda/include"]
        tmp = TENSOR_CALLS + ".tmp.%d" % os.getpid()
        subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-Wall", "-fPIC", "-shared", "-fvisibility=hidden",
                               "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, '-DBUILT_FOR="%s"' % torch.__version__,
                               "-I", sysconfig.get_paths()["include"], "-I", INCLUDE] + [x for h in headers for x in ("-isystem", h)] +
                              ["-o", tmp, TENSOR_CALLS_SOURCE, "-L", os.path.join(root, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu",
                               "-ltorch_python"])
        os.replace(tmp, TENSOR_CALLS)
    return TENSOR_CALLS


def build_library(force: bool = False, verbose: bool = False):
    """Returns the path of libavsg.so, rebuilding it (and the extension modules) when a source is newer.  The library needs no
    Python; where a module cannot be built (no C++ compiler, no Python.h, no torch) the binding goes without it."""
    lib = _build_library(force, verbose)
    for build in (build_calls, build_tensor_calls):
        try:
            build(force)
        except (ImportError, OSError, subprocess.CalledProcessError) as e:
            warnings.warn("an extension module of the binding was not built (%s): calls are marshalled by ctypes" % e)
    return lib


def _build_library(force: bool, verbose: bool):
    srcs = sources()
    if not srcs:
        return None
    if force or _stale(srcs):
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        tmp = LIB + ".tmp.%d" % os.getpid()
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-I", INCLUDE, "-I", CSRC,
                                                                               "-o", tmp] + srcs
        subprocess.check_call(cmd)
        os.replace(tmp, LIB)
    return LIB
