"""Builds libmoa_attn.so from csrc/ with nvcc for sm_103a, and the binding of PyTorch tensors to it,
moa_torch.so, with the host compiler (both in-tree, under _build/).  The library needs neither PyTorch
nor the binding; the binding belongs to the PyTorch that it was built against.

The translation units compile in parallel; the library links the CUDA
runtime statically and loads the driver's tensor-map encoder at run time, so it
has no link-time dependency on libcuda and loads on machines without a GPU.
"""
from __future__ import annotations

import concurrent.futures
import importlib.metadata
import importlib.util
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
BINDING_TORCH = BINDING + ".torch"   # which PyTorch it was built against
HEADERS = ["internal.h", "ops_internal.h", "kv4.cuh", "ptx.cuh", "tc_common.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xptxas", "-v"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found (set NVCC or put the CUDA toolkit on PATH)")


def _newest(names: list[str]) -> float:
    files = [os.path.join(CSRC, f) for f in names]
    files.append(os.path.join(HERE, "..", "include", "moa_attn.h"))
    files.append(os.path.abspath(__file__))
    return max(os.path.getmtime(f) for f in files)


def _fresh(path: str, names: list[str]) -> bool:
    return os.path.exists(path) and os.path.getmtime(path) >= _newest(names)


def _torch() -> str | None:
    """Which PyTorch a binding built now belongs to (None: there is none); nothing is imported."""
    spec = importlib.util.find_spec("torch")
    if spec is None or spec.origin is None:
        return None
    try:
        version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        version = "unknown"
    return "\n".join([version, spec.origin, sys.version])


def _binding_is_fresh(torch: str) -> bool:
    if not _fresh(BINDING, [BINDING_SOURCE]) or not os.path.exists(BINDING_TORCH):
        return False
    with open(BINDING_TORCH) as f:
        return f.read() == torch


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile (if stale) and return the path of libmoa_attn.so.

    The library is there before anything of the binding can fail.  Without PyTorch or a host compiler
    the binding is left out with a note; the operators that need it then raise at their first use."""
    os.makedirs(BUILD, exist_ok=True)
    torch = _torch()
    lib_stale = force or not _fresh(LIB, SOURCES + HEADERS)
    binding_stale = torch is not None and (force or not _binding_is_fresh(torch))
    if binding_stale and _cxx() is None:
        sys.stderr.write("moa_torch.so is left out: no host C++ compiler (set CXX or put g++ on PATH)\n")
        binding_stale = False
    elif torch is None and (lib_stale or not os.path.exists(BINDING)):
        sys.stderr.write("moa_torch.so is left out: PyTorch is not installed\n")
    with concurrent.futures.ThreadPoolExecutor(1) as ex:
        binding = ex.submit(_compile_binding) if binding_stale else None
        if lib_stale:
            _build_lib(verbose)
        if binding is not None:
            _link_binding(binding.result(), torch)
    return LIB


def _build_lib(verbose: bool) -> None:
    nvcc = _nvcc()

    def compile_one(src: str) -> tuple[str, str]:
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        cmd = [nvcc, *ARCH, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
        return obj, r.stderr

    with concurrent.futures.ThreadPoolExecutor(len(SOURCES)) as ex:
        results = list(ex.map(compile_one, SOURCES))
    if verbose:
        for _, log in results:
            sys.stderr.write(log)
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, "-shared", *ARCH, *[o for o, _ in results], "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)


def _run_cxx(cmd: list[str], what: str) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")


def _cxx() -> str | None:
    return os.environ.get("CXX") or shutil.which("g++") or shutil.which("c++")


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


def _link_binding(obj: str, made_for: str) -> None:
    import torch
    tmp = BINDING + f".tmp{os.getpid()}"
    _run_cxx([_cxx(), "-shared", obj, "-o", tmp, "-L", BUILD, "-l:libmoa_attn.so", "-Wl,-rpath,$ORIGIN",
              "-L", os.path.join(os.path.dirname(torch.__file__), "lib"),
              "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"], "linking the PyTorch binding")
    os.replace(tmp, BINDING)
    with open(BINDING_TORCH, "w") as f:
        f.write(made_for)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
