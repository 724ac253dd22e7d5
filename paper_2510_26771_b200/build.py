"""Build the CUDA library in-tree: csrc/*.cu -> paper_2510_26771_b200/libstamp.so (sm_100a only), and beside it the
Python module that marshals the block-scaled layers' calls: csrc/torch_calls.cpp -> _torch_calls.<torch and Python
version>.so (host code only).  The library alone, for callers in C, needs neither torch nor Python's headers."""
from __future__ import annotations

import os
import subprocess
import sys

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
_CSRC = os.path.join(_PKG, "csrc")
LIB_PATH = os.path.join(_PKG, "libstamp.so")


def _sources():
    srcs = [os.path.join(_CSRC, "stamp_api.cu")]
    deps = [os.path.join(_CSRC, f) for f in sorted(os.listdir(_CSRC)) if not f.endswith(".cpp")]
    return srcs, deps + [os.path.join(_ROOT, "include", "stamp.h")]


def _older(path: str, deps) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps)


def needs_build() -> bool:
    return _older(LIB_PATH, _sources()[1])


def calls_path() -> str:
    """The marshalling module for this torch and this Python: it is linked against both, so others get their own."""
    import sysconfig

    import torch
    return os.path.join(_PKG, f"_torch_calls.torch-{torch.__version__}.{sysconfig.get_config_var('SOABI')}.so")


def build_calls(force: bool = False) -> str:
    """Compile the marshalling module against torch's headers and the library (built before)."""
    import sysconfig

    import torch
    src, path = os.path.join(_CSRC, "torch_calls.cpp"), calls_path()
    if not force and not _older(path, [src, os.path.join(_ROOT, "include", "stamp.h")]):
        return path
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    tmp = path + f".tmp{os.getpid()}"
    try:
        subprocess.check_call(
            [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
             "-I", os.path.join(_ROOT, "include"), "-isystem", os.path.join(base, "include"),
             "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
             "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include"), "-o", tmp, src,
             "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda",
             "-L", _PKG, "-l:libstamp.so", "-Wl,-rpath,$ORIGIN"])
        os.replace(tmp, path)
    finally:
        if os.path.exists(tmp):
            os.remove(tmp)
    return path


def _calls_missing() -> str:
    """What the marshalling module would need and this machine lacks, or nothing."""
    import sysconfig
    try:
        import torch  # noqa: F401
    except ImportError:
        return "torch"
    return "" if os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")) else "Python.h"


def _build_calls_if_possible(force: bool) -> None:
    missing = _calls_missing()
    if missing:
        print(f"no {missing} here: the library is built, the marshalling module of the block-scaled calls is not (the "
              "binding raises where it is used)", file=sys.stderr)
    else:
        build_calls(force)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile with nvcc for sm_100a.  Returns the path of the shared library."""
    if not force and not needs_build():
        _build_calls_if_possible(False)
        return LIB_PATH
    srcs, _ = _sources()
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared",
           "-I", os.path.join(_ROOT, "include"), "-I", _CSRC, "-o", tmp] + srcs
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB_PATH)
    _build_calls_if_possible(force)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
