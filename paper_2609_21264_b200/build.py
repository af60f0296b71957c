"""Builds in-tree: the CUDA library with nvcc for sm_100a, which is all that the C ABI needs, and then, where torch is installed, the
extension module of the Python calls on drafted tokens with the C++ compiler (no JIT cache)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libfa_b200.so")
CALLS_PATH = os.path.join(_HERE, "_fa_calls.so")
CALLS_BUILT_FOR = os.path.join(_HERE, "_fa_calls.built")        # the Python and torch that the module was compiled against
SOURCES = ("fa_api.cu", "fa_noalloc.cu", "fa_paged.cu", "fa_drafts.cu", "fa_tree.cu", "fa_tree_few.cu")
NVCC_FLAGS = ("-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC", "-Xptxas", "-v", "--threads", "0")


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _newest_source_mtime() -> float:
    t = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(_HERE), "include")):
        for name in os.listdir(root):
            if name.endswith((".cu", ".cuh", ".h")):
                t = max(t, os.path.getmtime(os.path.join(root, name)))
    return t


def is_stale() -> bool:
    return (not os.path.exists(LIB_PATH)) or os.path.getmtime(LIB_PATH) < _newest_source_mtime()


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libfa_b200.so next to this file, and with torch the Python calls of csrc/fa_calls.cpp; returns the library's path."""
    if force or is_stale():
        _build_library(verbose)
    try:
        import torch  # noqa: F401
    except ImportError as e:
        warnings.warn("torch cannot be imported (%s): the extension module of the Python calls on drafted tokens is not built" % e)
    else:
        build_calls(force)
    return LIB_PATH


def _build_library(verbose: bool) -> None:
    tmp = LIB_PATH + ".tmp.%d" % os.getpid()
    extra = os.environ.get("FA_EXTRA_NVCC_FLAGS", "").split()
    cmd = [_nvcc(), *NVCC_FLAGS, *extra, "-o", tmp, *[os.path.join(CSRC, s) for s in SOURCES]]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    os.replace(tmp, LIB_PATH)
    if verbose:
        print(res.stdout + res.stderr)


def _built_for() -> str:
    try:
        with open(CALLS_BUILT_FOR) as f:
            return f.read()
    except OSError:
        return ""


def _running() -> str:
    """The Python and torch of this process, whose ABIs the extension module is linked against."""
    import torch
    return "%s, torch %s" % (sysconfig.get_config_var("SOABI"), torch.__version__)


def calls_mismatch() -> str:
    """What the extension module was built for, where that is not what runs; else an empty string (also where nothing says)."""
    built = _built_for()
    return built if built != _running() else ""


def build_calls(force: bool = False) -> str:
    """Compile csrc/fa_calls.cpp into the extension module _fa_calls.so next to this file, where its sources are newer or it was built for
    another Python or torch; returns its path."""
    import torch
    sources = max(os.path.getmtime(os.path.join(CSRC, "fa_calls.cpp")), os.path.getmtime(os.path.join(os.path.dirname(_HERE), "include", "fa.h")))
    if not force and os.path.exists(CALLS_PATH) and os.path.getmtime(CALLS_PATH) >= sources and _built_for() == _running():
        return CALLS_PATH
    root = os.path.dirname(torch.__file__)
    tmp = CALLS_PATH + ".tmp.%d" % os.getpid()
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    includes = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], cuda]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
           *["-I" + i for i in includes], "-o", tmp, os.path.join(CSRC, "fa_calls.cpp"), "-L" + os.path.join(root, "lib"),
           "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    if not shutil.which(cmd[0]):
        raise RuntimeError("%s not found" % cmd[0])
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("%s failed:\n" % cmd[0] + res.stdout + res.stderr)
    if os.path.exists(CALLS_BUILT_FOR):
        os.remove(CALLS_BUILT_FOR)              # (never a note beside another module than its own)
    os.replace(tmp, CALLS_PATH)
    with open(CALLS_BUILT_FOR, "w") as f:
        f.write(_running())
    return CALLS_PATH


if __name__ == "__main__":
    print(build(force=True, verbose=True))
