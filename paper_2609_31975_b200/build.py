"""Builds libsparse_ffn.so in-tree with nvcc for sm_100a (cross-compiles without a GPU).

Every source file is compiled to an object of its own (in parallel, only when it or a header changed) and the
objects are linked into the shared library.  `python -m paper_2609_31975_b200.build --trace` builds a second
library, libsparse_ffn_trace.so, whose single-token kernels write time stamps (see SFFN_KNOB_TRACE_BUFFER);
`--debug` builds libsparse_ffn_debug.so (-DSFFN_DEBUG), whose kernels check the indices they address global memory
with and report SFFN_ERR_BOUNDS in the device status instead of making the access.  Either is selected at run time
with the environment variable SFFN_LIBRARY."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libsparse_ffn.so"
CALLS = PKG / "_training.so"  # the training calls' Python side (csrc/torch_calls.cpp)
OBJ = PKG / "build"
SOURCES = ["api.cu", "general_kernels.cu", "fused_kernel.cu", "fused_tc_kernel.cu", "static_entry.cu",
           "batched_kernels.cu", "umma_kernels.cu", "cast_kernels.cu", "optim_kernels.cu", "train_simt.cu", "train_umma.cu", "train_umma_f32.cu", "train_join.cu", "train_outer.cu", "train_api.cu",
           "block_kernels.cu", "block_api.cu", "muon_kernels.cu", "muon_umma.cu", "muon_api.cu"]


def _headers_mtime() -> float:
    deps = list(CSRC.glob("*.cuh")) + list((ROOT / "include").glob("*.h"))
    return max(d.stat().st_mtime for d in deps)


def build_calls(force: bool = False) -> Path | None:
    """Compiles the module that checks and marshals the training calls' tensors, against the torch that is installed; again when that
    changes.  Where a compiler or headers for it are missing, which the C library does without, says so and leaves it out: the
    training calls from Python then raise."""
    import torch

    src = CSRC / "torch_calls.cpp"
    at, python, cxx = Path(torch.__file__).resolve().parent, Path(sysconfig.get_paths()["include"]), os.environ.get("CXX", "g++")
    made_for = f"torch {torch.__version__}, Python {sysconfig.get_python_version()}"
    stamp = OBJ / "_training.made_for"
    newest = max(src.stat().st_mtime, (ROOT / "include" / "sparse_ffn.h").stat().st_mtime)
    if not force and CALLS.exists() and CALLS.stat().st_mtime >= newest and stamp.exists() and stamp.read_text() == made_for:
        return CALLS
    missing = [str(f) for f in (python / "Python.h", at / "include" / "ATen" / "ATen.h") if not f.exists()] + ([] if shutil.which(cxx) else [cxx])
    if missing:
        CALLS.unlink(missing_ok=True)  # one made from other sources, or for another torch
        warnings.warn(f"{CALLS.name} is left out, and with it the training calls from Python: no {', '.join(missing)}")
        return None
    includes = [at / "include", at / "include" / "torch" / "csrc" / "api" / "include", python, Path(os.environ.get("CUDA_HOME", "/usr/local/cuda")) / "include"]
    tmp = CALLS.with_suffix(f".{os.getpid()}.tmp")
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f'-DSFFN_TORCH="{torch.__version__}"',
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", str(ROOT / "include")]
    for p in includes:
        cmd += ["-isystem", str(p)]
    cmd += [str(src), "-o", str(tmp), "-L", str(at / "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{src.name}:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, CALLS)
    OBJ.mkdir(parents=True, exist_ok=True)
    stamp.write_text(made_for)
    return CALLS


def build(force: bool = False, verbose: bool = False, trace: bool = False, debug: bool = False) -> Path:
    lib = build_library(force, verbose, trace, debug)
    build_calls(force)
    return lib


def build_library(force: bool = False, verbose: bool = False, trace: bool = False, debug: bool = False) -> Path:
    lib = PKG / "libsparse_ffn_trace.so" if trace else PKG / "libsparse_ffn_debug.so" if debug else LIB
    newest = max(_headers_mtime(), max((CSRC / s).stat().st_mtime for s in SOURCES))
    if not force and lib.exists() and lib.stat().st_mtime >= newest:
        return lib
    objdir = OBJ / ("trace" if trace else "debug" if debug else "plain")
    objdir.mkdir(parents=True, exist_ok=True)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
             "-I", str(ROOT / "include"), "-I", str(CSRC)]
    if trace:
        flags += ["-DSFFN_TRACE"]
    if debug:
        flags += ["-DSFFN_DEBUG"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    hdr = _headers_mtime()
    todo = []
    for s in SOURCES:
        src, obj = CSRC / s, objdir / (s + ".o")
        if force or not obj.exists() or obj.stat().st_mtime < max(src.stat().st_mtime, hdr):
            todo.append((src, obj))

    def compile_one(job):
        src, obj = job
        tmp = obj.with_suffix(f".{os.getpid()}.tmp")
        r = subprocess.run([nvcc, *flags, "-c", str(src), "-o", str(tmp)], capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src.name}:\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, obj)
        return r.stderr

    if todo:
        with ThreadPoolExecutor(max_workers=min(8, len(todo))) as pool:
            for log in pool.map(compile_one, todo):
                if verbose and log:
                    print(log, file=sys.stderr)
    objs = [objdir / (s + ".o") for s in SOURCES]
    if todo or not lib.exists() or any(o.stat().st_mtime > lib.stat().st_mtime for o in objs):
        tmp = lib.with_suffix(f".{os.getpid()}.tmp")
        subprocess.run([nvcc, "-shared", "-o", str(tmp), *map(str, objs)], check=True)
        os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, trace="--trace" in sys.argv, debug="--debug" in sys.argv))
