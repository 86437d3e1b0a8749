"""Builds libas_hybrid_attn.so in-tree with nvcc for sm_100a (cross-compiles without a GPU), and beside it as_torch_calls.so, the module of the calls that take
PyTorch tensors (csrc/torch_calls.cpp), with g++."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "lib", "libas_hybrid_attn.so")
TORCH_CALLS = os.path.join(PKG, "lib", "as_torch_calls.so")
BUILT_FOR = TORCH_CALLS + ".built_for"          # the PyTorch and Python that it was compiled against
SOURCES = ["as_hybrid_attn.cu", "simt_path.cu", "tensor_init.cu", "tensor_qpass.cu", "tensor_qstream.cu", "tensor_kpass.cu", "backward_simt.cu", "backward_tensor.cu", "backward_tensor_d64.cu", "no_alloc.cu",
           "block_rates.cu", "fp8_norm.cu", "fp8_matmul.cu"]


def _sources():
    return [os.path.join(CSRC, s) for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]


def _older(target: str, deps) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _headers():
    inc = os.path.join(ROOT, "include")
    return [os.path.join(inc, f) for f in os.listdir(inc) if f.endswith(".h")]


def _stale() -> bool:
    deps = _sources() + _headers()
    deps += [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    return _older(LIB, deps)


def torch_key() -> str:
    """What the module of the calls that take PyTorch tensors depends on beside its sources."""
    import torch
    return "torch %s, python %s" % (torch.__version__, sys.version.split()[0])


def _torch_calls_stale() -> bool:
    if _older(TORCH_CALLS, [os.path.join(CSRC, "torch_calls.cpp")] + _headers()) or not os.path.exists(BUILT_FOR):
        return True
    with open(BUILT_FOR) as f:
        return f.read() != torch_key()


def build_torch_calls(force: bool = False) -> str:
    """Compiles the module of the calls that take PyTorch tensors when it is missing, older than its source or made for another PyTorch or Python; returns its path."""
    if not force and not _torch_calls_stale():
        return TORCH_CALLS
    import sysconfig

    import torch
    source = os.path.join(CSRC, "torch_calls.cpp")
    libs, inc = (os.path.join(os.path.dirname(torch.__file__), d) for d in ("lib", "include"))
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include")]
    cmd += ["-isystem", inc, "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"), source, "-o", TORCH_CALLS, "-L", os.path.dirname(LIB), "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN",
            "-L", libs, "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-ltorch", "-lc10_cuda", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("%s failed:\n%s%s" % (cmd[0], res.stdout, res.stderr))
    with open(BUILT_FOR, "w") as f:
        f.write(torch_key())
    return TORCH_CALLS


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library, and the module beside it, where they are missing or older than their sources; returns the library's path."""
    if force or _stale():
        _build_library(verbose)
    build_torch_calls(force)
    return LIB


def _build_library(verbose: bool) -> None:
    os.makedirs(os.path.dirname(LIB), exist_ok=True)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads", "4",
           "--shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", LIB] + _sources()
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
