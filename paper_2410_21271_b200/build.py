"""Build libeora_linear.so (the C-ABI library) in-tree with nvcc for sm_100a, and _native.so (argument marshalling of the serving calls for Python).

Usage: python -m paper_2410_21271_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libeora_linear.so")
NATIVE = os.path.join(HERE, "_native.so")
SOURCES = ["eora_api.cu", "repack.cu", "generic.cu", "decode.cu", "decode_mid.cu", "decode_tc.cu", "tmat.cu", "prefill.cu", "noalloc.cu", "solve.cu", "solve_gemm.cu", "adapters.cu", "rotate.cu", "attention.cu"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _torch_dir() -> str:
    return os.path.dirname(importlib.util.find_spec("torch").origin)


def _native_flags() -> list:
    inc = os.path.join(_torch_dir(), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda", "include")
    return ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", f"-I{inc}", f"-I{os.path.join(inc, 'torch', 'csrc', 'api', 'include')}",
            f"-I{sysconfig.get_paths()['include']}", f"-I{cuda}"]


def needs_build() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(NATIVE):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(NATIVE))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "eora_linear.h"))
    deps.append(os.path.join(os.path.dirname(HERE), "include", "eora_solve.h"))
    deps.append(os.path.join(os.path.dirname(HERE), "include", "eora_serve.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    objs = []
    procs = []
    native = os.path.join(CSRC, "binding.o")
    procs.append(("binding.cpp", subprocess.Popen(["g++", *_native_flags(), "-c", os.path.join(CSRC, "binding.cpp"), "-o", native],
                                                  stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".cu", ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0:
            raise RuntimeError(f"compiler failed on {src}:\n{out}")
        if verbose and out:
            print(out)
    cmd = [_nvcc(), "-shared", "-o", LIB, *objs, "-lcudart"]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}")
    torch_lib = os.path.join(_torch_dir(), "lib")
    cmd = ["g++", "-shared", "-o", NATIVE, native, f"-L{HERE}", "-l:libeora_linear.so", "-Wl,-rpath,$ORIGIN", f"-L{torch_lib}", f"-Wl,-rpath,{torch_lib}",
           "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
