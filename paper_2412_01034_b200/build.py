"""Builds ``libqil.so`` (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libqil.so")
BINDING = os.path.join(HERE, "_qil_torch.so")
BINDING_SOURCE = "torch_binding.cpp"
SOURCES = ["api.cu", "quantize.cu", "w4a16_general.cu", "w4a16_skinny.cu", "w4a4.cu", "ref_gemv.cu",
           "w4a16_static_ws.cu", "w4a16_tc.cu", "w4a16_prefill.cu", "w8a16.cu", "probe_mma.cu", "igemm_list.cu", "lora_side.cu",
           "rmsnorm.cu", "rope_cache.cu", "attn_paged.cu", "attn_few.cu", "attn_many.cu", "lora_batch.cu"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _older(out: str, deps) -> bool:
    return not os.path.exists(out) or any(os.path.getmtime(d) > os.path.getmtime(out) for d in deps)


def needs_build() -> bool:
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != BINDING_SOURCE] + [os.path.join(ROOT, "include", "qil.h")]
    return _older(OUT, deps)


def build_binding(force: bool = False) -> str:
    """The Python marshalling of the layer operators (C++, against the installed torch's headers)."""
    source, header = os.path.join(CSRC, BINDING_SOURCE), os.path.join(ROOT, "include", "qil.h")
    if not force and not _older(BINDING, [source, header]):
        return BINDING
    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    includes = [os.path.join(ROOT, "include"), sysconfig.get_paths()["include"], os.path.join(base, "include"),
                os.path.join(base, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [f"-isystem{i}" for i in includes] + [source, "-o", BINDING, "-L", os.path.join(base, "lib"), "-L", HERE, "-l:libqil.so",
                                                 "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ltorch_cuda", "-Wl,-rpath,$ORIGIN"]
    subprocess.run(cmd, check=True)
    return BINDING


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        build_binding()
        return OUT
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", OUT] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.run(cmd, check=True)
    build_binding(force)
    return OUT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
