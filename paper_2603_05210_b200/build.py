"""Builds ``libvt.so`` (the CUDA library behind ``include/vt.h``) in-tree with nvcc for sm_100a, and ``_vt_torch.so``, the compiled
marshalling of torch tensors for some of its calls, with the host compiler."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libvt.so")
MARSHAL = os.path.join(HERE, "_vt_torch.so")
SOURCES = ["vt_api.cu", "vt_attn.cu", "vt_aux.cu", "vt_ffn.cu", "vt_gemm.cu", "vt_head_gemv.cu", "vt_head_mma.cu", "vt_head_mma_small.cu",
           "vt_merge.cu", "vt_probe.cu", "vt_rope.cu", "vt_score.cu", "vt_score_grad.cu", "vt_select.cu", "vt_verify.cu"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


MARSHAL_SOURCE = "vt_torch.cpp"


def _newer(target: str, sources) -> bool:
    paths = [os.path.join(CSRC, f) for f in sources] + [os.path.join(HERE, "..", "include", "vt.h")]
    return os.path.exists(target) and os.path.getmtime(target) >= max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    """``build_library`` and ``build_marshal`` side by side."""
    with ThreadPoolExecutor(max_workers=1) as pool:
        marshal = pool.submit(build_marshal, force)
        lib = build_library(force, verbose)
        marshal.result()
    return lib


def build_marshal(force: bool = False) -> str:
    """Compile ``vt_torch.cpp`` against the installed PyTorch; a no-op when ``_vt_torch.so`` is newer than its source."""
    if not force and _newer(MARSHAL, [MARSHAL_SOURCE]):
        return MARSHAL
    import torch
    root, cuda = os.path.dirname(torch.__file__), os.path.dirname(os.path.dirname(shutil.which(os.environ.get("NVCC", "nvcc")) or "/usr/local/cuda/bin/nvcc"))
    tmp = MARSHAL + f".{os.getpid()}.tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           *(a for d in (sysconfig.get_paths()["include"], f"{root}/include", f"{root}/include/torch/csrc/api/include", f"{cuda}/include")
             for a in ("-isystem", d)),
           os.path.join(CSRC, MARSHAL_SOURCE), "-o", tmp, f"-L{root}/lib", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed for {MARSHAL_SOURCE}:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, MARSHAL)
    return MARSHAL


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every ``.cu`` under ``csrc/`` and link ``libvt.so``; a no-op when the library is newer than its sources."""
    if not force and _newer(LIB, [f for f in os.listdir(CSRC) if f != MARSHAL_SOURCE]):
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    os.makedirs(OBJ, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose else []

    def compile_one(src):
        obj = os.path.join(OBJ, src.replace(".cu", ".o"))
        cmd = [nvcc, *NVCC_FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    tmp = LIB + f".{os.getpid()}.tmp"
    r = subprocess.run([nvcc, "-shared", "-o", tmp, *objs, "-lcudart"], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
