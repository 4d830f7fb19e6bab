"""Compile the CUDA library in-tree for sm_100a: ``python -m paper_2602_01901_b200.build``."""

from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libqcache.so")
EXTENSION = os.path.join(HERE, "_qc_torch.so")
SOURCES = ["qc_runtime.cu", "qc_kernels.cu", "qc_attend_tc.cu", "qc_rows.cu", "qc_prefill.cu", "qc_calib.cu", "qc_static.cu",
           "qc_table.cu", "qc_quant.cu", "qc_quant_attend.cu"]
HEADERS = ["qc_internal.h", "qc_device.cuh", "qc_quant.h", "qc_quant.cuh", os.path.join("..", "..", "include", "qc.h")]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _older(target: str, sources) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(os.path.join(CSRC, s)) > t for s in sources)


def is_stale() -> bool:
    return _older(LIB, SOURCES + HEADERS)


def built_for() -> str:
    """The torch and Python whose binary interface a module of theirs has."""
    import torch

    return f"torch {torch.__version__}, Python {sys.version_info[0]}.{sys.version_info[1]}"


def _extension_is_stale() -> bool:
    if _older(EXTENSION, ["qc_torch.cpp", os.path.join("..", "..", "include", "qc.h")]):
        return True
    with open(EXTENSION, "rb") as f:
        return f"_qc_torch for {built_for()};".encode() not in f.read()      # (what qc_torch.cpp holds of QC_BUILT_FOR)


def _lacking() -> str:
    """What the extension needs and this machine does not have (nothing: it can be built)."""
    import sysconfig

    try:
        import torch  # noqa: F401
        from torch.utils import cpp_extension
    except ImportError as e:
        return str(e)
    if not shutil.which("g++"):
        return "no g++"
    for path, name in ((sysconfig.get_paths()["include"], "Python.h"), (cpp_extension.include_paths()[0], os.path.join("ATen", "ATen.h"))):
        if not os.path.exists(os.path.join(path, name)):
            return f"no {name} in {path}"
    return ""


def _build_extension() -> None:
    """The Python module that takes torch tensors to the library (host code only)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    where = os.path.join(os.path.dirname(torch.__file__), "lib")
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DQC_BUILT_FOR="{built_for()}"']
    for path in [*cpp_extension.include_paths(), os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", path]
    cmd += ["-o", EXTENSION, os.path.join(CSRC, "qc_torch.cpp"), "-L" + HERE, "-l:libqcache.so", "-Wl,-rpath,$ORIGIN", "-L" + where, "-lc10", "-lc10_cuda",
            "-ltorch_cpu", "-ltorch_python"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds what is out of date.  The library needs nvcc alone; where torch's or Python's headers are missing, the module behind
    ``quant`` is left out, with a line on stderr (``quant`` says so itself when it is used)."""
    if force or is_stale():
        cmd = [
            _nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
            "-Xcompiler", "-fPIC", "-shared", "-o", LIB,
        ] + [os.path.join(CSRC, s) for s in SOURCES]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        res = subprocess.run(cmd, capture_output=True, text=True)
        if verbose:
            sys.stderr.write(res.stderr)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    lacking = _lacking()
    if lacking:
        sys.stderr.write(f"{EXTENSION} is not built ({lacking}): the calls of quant.py need it\n")
    elif force or _extension_is_stale():
        _build_extension()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
