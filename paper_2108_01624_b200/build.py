"""Builds libdp_b200.so (sm_100a, nvcc) and the CPython module _dp_tensors.so (g++) in-tree.  `python -m paper_2108_01624_b200.build`."""
from __future__ import annotations

import os
import subprocess
import sys
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdp_b200.so")
HEADER = os.path.join(HERE, "..", "include", "dp.h")
MODULE = os.path.join(HERE, "_dp_tensors.so")          # CPython module: torch tensors into the C ABI
SOURCES = ["dp_api.cu", "dp_stream.cu", "dp_generic.cu", "dp_umma.cu", "dp_noalloc.cu",
           "dp_clip.cu", "dp_rows.cu", "dp_relpos.cu", "dp_qknorm.cu"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _older(path: str, *deps: str) -> bool:
    """`path` is missing, or older than one of `deps` or than this file (the build commands)."""
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in (*deps, __file__))


def needs_library() -> bool:
    return _older(LIB, HEADER, *(os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")))


def module_key() -> str:
    """What _dp_tensors.so is compiled against: it reads tensors through torch's C++ headers and Python's."""
    import sysconfig

    import torch
    return (f"_dp_tensors for torch {torch.__version__}, C++11 ABI {int(torch._C._GLIBCXX_USE_CXX11_ABI)}, "
            f"{sysconfig.get_config_var('SOABI')}")


def module_fits(path: str = MODULE) -> bool:
    """The module at `path` was built for the installed torch and the running Python (whose key it carries)."""
    with open(path, "rb") as f:
        return module_key().encode() + b"\0" in f.read()


def needs_module() -> bool:
    return _older(MODULE, HEADER, os.path.join(CSRC, "dp_tensors.cpp")) or not module_fits(MODULE)


def needs_build() -> bool:
    return needs_library() or needs_module()


def build(force: bool = False, verbose: bool = False, defines=(), out: str = LIB) -> str:
    """Compile every .cu for sm_100a into one shared library next to this file (or `out`, with extra -D flags)."""
    if out != LIB or defines or force or needs_library():
        _build_library(verbose, defines, out)
    if out == LIB and (force or needs_module()):
        try:
            build_module()
        except RuntimeError as e:          # the C ABI and the calls bound by ctypes are complete without it
            warnings.warn(f"_dp_tensors.so was not built, the calls on small tensors will raise ImportError: {e}",
                          RuntimeWarning, stacklevel=2)
    return out


def _build_library(verbose: bool, defines, out: str) -> None:
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--threads", "8",
           "-I", os.path.join(HERE, "..", "include")]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [f"-D{d}" for d in defines]
    cmd += [os.path.join(CSRC, s) for s in SOURCES] + ["-o", out]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + proc.stdout + proc.stderr)
    if verbose:
        print(proc.stderr)


def build_module() -> str:
    """The CPython module, host code only, against the installed torch's headers.  Raises RuntimeError where a compiler or
    headers are missing; no older module is left then."""
    import sysconfig

    import torch
    base = os.path.dirname(os.path.abspath(torch.__file__))
    cuda = os.path.dirname(os.path.dirname(os.path.abspath(_nvcc()))) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    if os.path.exists(MODULE):
        os.remove(MODULE)
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DDP_MODULE_KEY="{module_key()}"',
           "-isystem", os.path.join(base, "include"), "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include"),
           os.path.join(CSRC, "dp_tensors.cpp"), "-o", MODULE, "-L", os.path.join(base, "lib"),
           "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", f"-Wl,-rpath,{os.path.join(base, 'lib')}"]
    try:
        proc = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError(f"{cmd[0]}: {e}") from e
    if proc.returncode != 0:
        raise RuntimeError("g++ failed:\n" + proc.stdout + proc.stderr)
    return MODULE


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
