"""Builds libtq.so (host C++ + CUDA sm_100a) in-tree with nvcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sysconfig
import warnings
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libtq.so"
FAST_SOURCE = CSRC / "tq_fast.cpp"  # CPython module: the usual case of the calls between the linear layers
SOURCES = [CSRC / "tq_device.cu", CSRC / "tq_gemm.cu", CSRC / "tq_gemm_ws.cu", CSRC / "tq_tiles.cu", CSRC / "tq_wide.cu", CSRC / "tq_encode.cu", CSRC / "tq_dict_device.cu",
           CSRC / "tq_norm.cu", CSRC / "tq_rope.cu", CSRC / "tq_attn.cu", CSRC / "tq_cross.cu", CSRC / "tq_host.cpp"]
HEADERS = [CSRC / "tq_internal.h", CSRC / "tq_sm100.cuh", CSRC / "tq_tiles_common.cuh", CSRC / "tq_ops_common.cuh", ROOT / "include" / "tq.h"]


def _nvcc() -> str | None:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    return cand if os.path.exists(cand) else None


def is_stale() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    return any(p.stat().st_mtime > t for p in SOURCES + HEADERS if p.exists())


def build_library(force: bool = False, verbose: bool = False) -> Path:
    # a prebuilt library elsewhere (deployments without nvcc): TQ_LIBTQ=/path/to/libtq.so
    prebuilt = os.environ.get("TQ_LIBTQ")
    if prebuilt and not force:
        if not os.path.exists(prebuilt):
            raise RuntimeError(f"TQ_LIBTQ={prebuilt} does not exist")
        return Path(prebuilt)
    if not force and not is_stale():
        return LIB
    nvcc = _nvcc()
    if nvcc is None:
        raise RuntimeError("libtq.so is missing or stale and nvcc was not found; cannot build the CUDA library")
    tmp = LIB.with_name(f"libtq.tmp{os.getpid()}.so")
    cmd = [nvcc, "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "--threads", "8", "-Xcompiler", "-fPIC,-O3,-pthread", "-shared", "-I", str(ROOT / "include"), "-I", str(CSRC),
           "-o", str(tmp)] + [str(s) for s in SOURCES] + ["-lpthread"]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


def fast_path() -> Path:
    """Where the CPython module lies: it is built against one interpreter and one torch, and its name says which."""
    import torch
    return PKG / f"_tqfast.{sysconfig.get_config_var('SOABI')}.torch-{torch.__version__}.so"


def build_fast(force: bool = False) -> Path | None:
    """Builds the CPython module; None where that is not possible (no compiler, no headers of the running interpreter or of torch, a
    dlpack.h without the exchange interface, a folder that cannot be written): binding.py does without.  force: raises instead where
    the compiler fails."""
    import torch
    fast = fast_path()
    sources = [FAST_SOURCE, ROOT / "include" / "tq.h"]
    if not force and fast.exists() and fast.stat().st_mtime >= max(p.stat().st_mtime for p in sources):
        return fast
    python, dlpack = Path(sysconfig.get_paths()["include"]), Path(torch.__file__).parent / "include"
    gxx = shutil.which("g++")
    if gxx is None or not (python / "Python.h").exists() or not (dlpack / "ATen" / "dlpack.h").exists():
        return None
    tmp = PKG / f"_tqfast.tmp{os.getpid()}.so"
    cmd = [gxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", str(ROOT / "include"), "-I", str(python), "-I", str(dlpack), str(FAST_SOURCE), "-o", str(tmp)]
    try:
        subprocess.run(cmd, check=True, stderr=None if force else subprocess.PIPE)
        os.replace(tmp, fast)
    except (subprocess.CalledProcessError, OSError) as e:
        tmp.unlink(missing_ok=True)
        if force:
            raise
        warnings.warn(f"the native form of the small calls was not built, they go through Python: {e}", RuntimeWarning, stacklevel=2)
        return None
    return fast


if __name__ == "__main__":
    import sys
    build_fast(force=True)
    print(build_library(force=True, verbose="-v" in sys.argv))
