"""Builds libmoa_attn.so from csrc/ with nvcc for sm_103a, and the binding of PyTorch tensors to it,
moa_torch.so, with the host compiler (both in-tree, under _build/).

The translation units compile in parallel; the library links the CUDA
runtime statically and loads the driver's tensor-map encoder at run time, so it
has no link-time dependency on libcuda and loads on machines without a GPU.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libmoa_attn.so")
SOURCES = ["moa_attn_api.cu", "attn_fwd_f32_cc.cu", "attn_fwd_bf16_tc.cu", "attn_bwd_bf16_tc.cu",
           "attn_bwd_f32_cc.cu", "qkv_proj_bf16_tc.cu", "moa_ops_api.cu", "qk_norm_rope.cu",
           "kv4_cache.cu", "kv4_attn.cu", "kv4_attn_tc.cu"]
BINDING = os.path.join(BUILD, "moa_torch.so")
BINDING_SOURCE = "torch_binding.cpp"
HEADERS = ["internal.h", "ops_internal.h", "kv4.cuh", "ptx.cuh", "tc_common.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found (set NVCC or put the CUDA toolkit on PATH)")


def _newest_input() -> float:
    files = [os.path.join(CSRC, f) for f in SOURCES + HEADERS + [BINDING_SOURCE]]
    files.append(os.path.join(HERE, "..", "include", "moa_attn.h"))
    files.append(os.path.abspath(__file__))
    return max(os.path.getmtime(f) for f in files)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile (if stale) and return the path of libmoa_attn.so."""
    os.makedirs(BUILD, exist_ok=True)
    done = [f for f in (LIB, BINDING) if os.path.exists(f)]
    if not force and len(done) == 2 and min(map(os.path.getmtime, done)) >= _newest_input():
        return LIB
    nvcc = _nvcc()

    def compile_one(src: str) -> tuple[str, str]:
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        cmd = [nvcc, *ARCH, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
        return obj, r.stderr

    with concurrent.futures.ThreadPoolExecutor(len(SOURCES) + 1) as ex:
        binding = ex.submit(_compile_binding)
        results = list(ex.map(compile_one, SOURCES))
        binding = binding.result()
    if verbose:
        for _, log in results:
            sys.stderr.write(log)
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, "-shared", *ARCH, *[o for o, _ in results], "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    _link_binding(binding)
    return LIB


def _run_cxx(cmd: list[str], what: str) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")


def _cxx() -> str:
    cxx = os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")
    if not cxx:
        raise RuntimeError("no host C++ compiler found (set CXX or put g++ on PATH)")
    return cxx


def _compile_binding() -> str:
    """Object file of the PyTorch binding (needs the headers that PyTorch installs)."""
    import torch
    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    obj = os.path.join(BUILD, "torch_binding.o")
    _run_cxx([_cxx(), "-std=c++17", "-O2", "-fPIC", "-fvisibility=hidden",
              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
              "-isystem", inc, "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"),
              "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include"),
              "-c", os.path.join(CSRC, BINDING_SOURCE), "-o", obj], "compiling the PyTorch binding")
    return obj


def _link_binding(obj: str) -> None:
    import torch
    tmp = BINDING + f".tmp{os.getpid()}"
    _run_cxx([_cxx(), "-shared", obj, "-o", tmp, "-L", BUILD, "-l:libmoa_attn.so", "-Wl,-rpath,$ORIGIN",
              "-L", os.path.join(os.path.dirname(torch.__file__), "lib"),
              "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"], "linking the PyTorch binding")
    os.replace(tmp, BINDING)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
