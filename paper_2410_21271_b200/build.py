"""Build libeora_linear.so (the C-ABI library) in-tree with nvcc for sm_100a, and, where there is a torch with CUDA, _native.so (argument marshalling of the serving calls for Python).

Usage: python -m paper_2410_21271_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import importlib.util
import os
import re
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libeora_linear.so")
NATIVE = os.path.join(HERE, "_native.so")
SOURCES = ["eora_api.cu", "repack.cu", "generic.cu", "decode.cu", "decode_mid.cu", "decode_tc.cu", "tmat.cu", "prefill.cu", "noalloc.cu", "solve.cu", "solve_gemm.cu", "adapters.cu", "rotate.cu", "attention.cu"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _torch_dir():
    """torch's folder; None where there is no torch, or one without CUDA."""
    spec = importlib.util.find_spec("torch")
    where = os.path.dirname(spec.origin) if spec is not None and spec.origin else None
    return where if where and os.path.exists(os.path.join(where, "lib", "libc10_cuda.so")) else None


def _built_for(torch_dir: str) -> str:
    """What _native.so goes with; the module carries it as its documentation."""
    with open(os.path.join(torch_dir, "version.py")) as f:
        found = re.search(r"__version__\s*=\s*['\"]([^'\"]+)", f.read())
    return f"torch {found.group(1) if found else '?'}, {sys.implementation.cache_tag}"


def _native_flags(torch_dir: str) -> list:
    inc = os.path.join(torch_dir, "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())) or "/usr/local/cuda", "include")
    return ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", f'-DEORA_BUILT_FOR="{_built_for(torch_dir)}"', f"-I{inc}",
            f"-I{os.path.join(inc, 'torch', 'csrc', 'api', 'include')}", f"-I{sysconfig.get_paths()['include']}", f"-I{cuda}"]


def _older(target: str, deps) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _library_needs_build() -> bool:
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))]
    return _older(LIB, deps + [os.path.join(INCLUDE, f"eora_{h}.h") for h in ("linear", "solve", "serve")])


def _native_needs_build() -> bool:
    """Where there is no torch, never: the library does without."""
    where = _torch_dir()
    if where is None:
        return False
    if _older(NATIVE, [os.path.join(CSRC, "binding.cpp")] + [os.path.join(INCLUDE, f"eora_{h}.h") for h in ("linear", "serve")]):
        return True
    with open(NATIVE, "rb") as f:
        return _built_for(where).encode() not in f.read()


def needs_build() -> bool:
    return _library_needs_build() or _native_needs_build()


def _finish(procs, verbose: bool) -> None:
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0:
            raise RuntimeError(f"compiler failed on {src}:\n{out}")
        if verbose and out:
            print(out)


def _link(cmd) -> None:
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}")


def _start(cmd):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def build(force: bool = False, verbose: bool = False) -> str:
    """The library, which needs nvcc alone, and, where there is a torch with CUDA, the marshalling for it."""
    where = _torch_dir()
    library, native = force or _library_needs_build(), where is not None and (force or _native_needs_build())
    objs, procs = [], []
    if library:
        for src in SOURCES:
            objs.append(os.path.join(CSRC, src.replace(".cu", ".o")))
            procs.append((src, _start([_nvcc(), *(["-Xptxas=-v"] if verbose else []), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", objs[-1]])))
    binding = os.path.join(CSRC, "binding.o")
    native_procs = [("binding.cpp", _start(["g++", *_native_flags(where), "-c", os.path.join(CSRC, "binding.cpp"), "-o", binding]))] if native else []
    _finish(procs, verbose)
    if library:
        _link([_nvcc(), "-shared", "-o", LIB, *objs, "-lcudart"])
    _finish(native_procs, verbose)
    if native:
        torch_lib = os.path.join(where, "lib")
        _link(["g++", "-shared", "-o", NATIVE, binding, f"-L{HERE}", "-l:libeora_linear.so", "-Wl,-rpath,$ORIGIN", f"-L{torch_lib}", f"-Wl,-rpath,{torch_lib}",
               "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"])
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
