"""Build the HIP library (csrc/*.hip -> libzc.so) for gfx950 with hipcc, and the native calls of the binding for this Python, in-tree."""
import importlib.util
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libzc.so")
SOURCES = ["zc_api.hip", "zc_layers.hip"]
CALLS = os.path.join(HERE, "_zc_calls" + sysconfig.get_config_var("EXT_SUFFIX"))      # (named for this Python: another one leaves it alone)
LAYER_CALLS = os.path.join(HERE, "_zc_layer_calls" + sysconfig.get_config_var("EXT_SUFFIX"))

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++20", "-fPIC", "-shared",
    "-ffp-contract=off",                                     # quantisation is defined by separate roundings
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-mllvm", "-amdgpu-kernarg-preload-count=16",            # a kernel's leading scalar arguments are in registers when a wave starts
    "-Wall", "-Wno-unused-function",
]


def build_all(verbose=False, extra=()):
    """The library and all native calls of the binding."""
    build(verbose, extra)
    build_layer_calls(verbose)
    return LIB


def build(verbose=False, extra=()):
    """The library and the codec's native calls: what needs nothing of torch."""
    cmd = ["hipcc", *FLAGS, *extra, *[os.path.join(CSRC, s) for s in SOURCES], "-o", LIB]
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)
    build_calls(verbose)
    return LIB


def build_calls(verbose=False):
    """The native calls, which the binding does without where they are missing: they need the headers of this Python and a C++ compiler."""
    _build_module(CALLS, ["zc_calls.cpp"], verbose)


def build_layer_calls(verbose=False):
    """Those that read torch's tensors, a module of its own: they need torch's headers and libraries besides."""
    if os.path.exists(LAYER_CALLS):
        os.remove(LAYER_CALLS)
    spec = importlib.util.find_spec("torch")
    home = os.path.dirname(spec.origin) if spec and spec.origin else ""
    headers, libraries = os.path.join(home, "include"), os.path.join(home, "lib")
    if not os.path.exists(os.path.join(headers, "torch", "csrc", "autograd", "python_variable.h")) or not os.path.exists(os.path.join(libraries, "libtorch_python.so")):
        print("no headers of torch: the layer calls go through ctypes")
        return
    _build_module(LAYER_CALLS, ["zc_layer_calls.cpp"], verbose, "-isystem", headers, "-isystem", os.path.join(headers, "torch", "csrc", "api", "include"),
                  "-L" + libraries, "-ltorch_python", "-ltorch_cpu", "-lc10")


def _build_module(to, sources, verbose, *more):
    include = sysconfig.get_paths()["include"]
    if os.path.exists(to):
        os.remove(to)                                        # (not one of other sources beside the library)
    if not os.path.exists(os.path.join(include, "Python.h")) or not shutil.which("g++"):
        print("no headers of this Python or no g++: the binding goes through ctypes alone")
        return
    cmd = ["g++", "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-I" + include, *[os.path.join(CSRC, s) for s in sources], *more, "-o", to]
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)


if __name__ == "__main__":
    print(build_all(verbose=True))
