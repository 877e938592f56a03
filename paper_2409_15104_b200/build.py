"""Build libpec.so (the C-ABI library) for sm_100a with nvcc, and _pec_torch.so (tensor marshalling for binding.py), in-tree."""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libpec.so")
TORCH_SOURCE = "pec_torch.cpp"
TORCH_MODULE = os.path.join(HERE, "_pec_torch.so")
SOURCES = ["pec_api.cpp", "pec_plan.cpp", "pec_merge.cu", "pec_attn_f32.cu", "pec_attn_prefill_bf16.cu", "pec_attn_split_bf16.cu", "pec_decode.cu", "pec_linear.cu", "pec_linear_merged.cu",
           "pec_heads.cu", "pec_paged_attn.cu", "pec_paged_few.cu", "pec_paged_many.cu"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != TORCH_SOURCE] + [os.path.join(INCLUDE, "pec.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def _build_torch_module(force: bool) -> None:
    import torch
    # Beside the module: what it was built for.  One built for another torch or Python does not load, whatever its age.
    mark = os.path.join(os.path.dirname(TORCH_MODULE), "_pec_torch.built_for")
    built_for = f"torch {torch.__version__}, Python {sys.version}"
    deps = [os.path.join(CSRC, TORCH_SOURCE), os.path.join(INCLUDE, "pec.h")]
    if not force and os.path.exists(TORCH_MODULE) and all(os.path.getmtime(d) <= os.path.getmtime(TORCH_MODULE) for d in deps):
        if os.path.exists(mark):
            with open(mark) as f:
                if f.read() == built_for:
                    return
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    includes = [INCLUDE, os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
                os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for d in includes:
        cmd += ["-isystem" if d != INCLUDE else "-I", d]
    cmd += [os.path.join(CSRC, TORCH_SOURCE), "-o", TORCH_MODULE, "-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu",
            "-ltorch_cuda", "-lc10", "-lc10_cuda"]
    subprocess.run(cmd, check=True)
    with open(mark, "w") as f:
        f.write(built_for)


def _build_library(verbose: bool) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC, "-o", LIB]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.run(cmd, check=True)


def build(force: bool = False, verbose: bool = False) -> str:
    # The C library first: it needs neither torch nor g++, and is there for C callers where the module cannot be built.
    if force or _stale():
        _build_library(verbose)
    _build_torch_module(force)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
