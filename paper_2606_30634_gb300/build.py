"""Build the package's native libraries in-tree for sm_103a.

* ``_build/libdpo.so``       -- the product: C ABI of include/dpo.h and its
                                kernels (csrc/).
* ``_build/dpo_tensors.so``   -- the feed-forward calls on PyTorch tensors, a
                                Python module (ffn.py's other half), compiled
                                against PyTorch's headers by the host compiler.
* ``_build/libdpo_synth.so`` -- seeded synthetic inputs (include/dpo_synth.h),
                                used by the tests and the benchmark.

Each translation unit compiles in its own nvcc process (in parallel), then one
link per library. Rebuilds only what is older than its sources.
``python -m paper_2606_30634_gb300.build [--force]``.
"""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
INCLUDE = os.path.join(ROOT, "include")
OUT = os.path.join(PKG, "_build")
NVCC = os.environ.get("NVCC", "nvcc")
CXX = os.environ.get("CXX", "g++")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
COMMON = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-O3,-fopenmp",
                 "-I", INCLUDE]

LIBS = {
    "libdpo.so": {
        "sources": ["csrc/dpo_kernels.cu", "csrc/dpo_step_adamw.cu", "csrc/dpo_step_nadam.cu",
                    "csrc/dpo_step_lion.cu", "csrc/dpo_step_adan.cu", "csrc/dpo_abi.cpp",
                    "csrc/dpo_noalloc.cu", "csrc/dpo_muon.cu", "csrc/dpo_rmsnorm.cu",
                    "csrc/dpo_ffn.cu"],
        "headers": ["csrc/dpo_internal.h", "csrc/dpo_device.cuh", "csrc/dpo_reduce.cuh",
                    "csrc/dpo_step.cuh",
                    "csrc/dpo_gemm.cuh", "csrc/dpo_call.h", "csrc/dpo_pack8.cuh",
                    "csrc/dpo_ffn_gemm.cuh", "csrc/dpo_ffn_few.cuh", "../include/dpo.h",
                    "../include/dpo_muon.h"],
        "includes": ["csrc"],
        "ptxas_v": ["csrc/dpo_step_adamw.cu", "csrc/dpo_muon.cu", "csrc/dpo_ffn.cu"],
    },
    "dpo_tensors.so": {
        "sources": ["csrc/dpo_tensors.cpp"],
        "headers": ["../include/dpo.h"],
        "includes": [],
        "ptxas_v": [],
        "torch": True,
    },
    "libdpo_synth.so": {
        "sources": ["synth/synth.cu"],
        "headers": ["synth/philox.h", "../include/dpo_synth.h"],
        "includes": ["synth"],
        "ptxas_v": [],
    },
}


def _mtime(p):
    return os.path.getmtime(p) if os.path.exists(p) else -1.0


def _torch_flags():
    """(compile flags, link flags) of a Python module that uses PyTorch's C++ interface."""
    import sysconfig
    import torch
    root = os.path.dirname(torch.__file__)
    nvcc = shutil.which(NVCC) or "/usr/local/cuda/bin/nvcc"
    inc = [os.path.join(root, "include"), sysconfig.get_paths()["include"],
           os.path.join(os.path.dirname(os.path.dirname(nvcc)), "include")]
    lib = os.path.join(root, "lib")
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    return (["-O2", "-std=c++17", "-fPIC", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={abi}", "-I", INCLUDE] +
            sum((["-isystem", i] for i in inc), []),
            ["-shared", "-L" + lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch_cpu", "-lc10",
             "-lc10_cuda"])


def _torch_tag() -> str:
    """What a module built against PyTorch depends on beside its sources."""
    import torch
    return f"python {sys.version}\ntorch {torch.__version__} in {os.path.dirname(torch.__file__)}\n"


def _read(path):
    if not os.path.exists(path):
        return None
    with open(path) as f:
        return f.read()


def _run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")
    return r.stderr


def _compile(src, obj, includes, verbose_ptxas, torch=False):
    if torch:
        return _run([CXX] + _torch_flags()[0] + ["-c", os.path.join(PKG, src), "-o", obj],
                    f"{CXX} for {src}")
    cmd = [NVCC] + COMMON + sum((["-I", os.path.join(PKG, i)] for i in includes), [])
    if src.endswith(".cpp"):
        cmd += ["-x", "cu"]
    if verbose_ptxas:
        cmd += ["-Xptxas", "-v"]
    cmd += ["-c", os.path.join(PKG, src), "-o", obj]
    return _run(cmd, f"nvcc for {src}")


def build(force: bool = False, quiet: bool = True, only=None) -> dict:
    """Compile every library whose sources changed, or those of ``only``; returns
    {name: path}. A library's user builds that one alone: the optimizers need no Python
    headers, which dpo_tensors.so does."""
    os.makedirs(OUT, exist_ok=True)
    names = list(LIBS if only is None else only)
    jobs = []
    for lib in names:
        spec = LIBS[lib]
        out = os.path.join(OUT, lib)
        deps = [os.path.join(PKG, p) for p in spec["sources"] + spec["headers"]]
        other = spec.get("torch", False) and _read(out + ".tag") != _torch_tag()
        if force or other or any(_mtime(d) > _mtime(out) for d in deps):
            for src in spec["sources"]:
                obj = os.path.join(OUT, os.path.basename(src) + ".o")
                jobs.append((lib, src, obj, spec["includes"], src in spec["ptxas_v"],
                             spec.get("torch", False)))
    if jobs:
        with ThreadPoolExecutor(max_workers=max(1, min(len(jobs), os.cpu_count() or 1))) as ex:
            logs = list(ex.map(lambda j: _compile(*j[1:]), jobs))
        if not quiet:
            for j, log in zip(jobs, logs):
                if log.strip():
                    print(f"[{j[1]}]\n{log}", file=sys.stderr)
        for lib in sorted({j[0] for j in jobs}):
            objs = [os.path.join(OUT, os.path.basename(s) + ".o") for s in LIBS[lib]["sources"]]
            out = os.path.join(OUT, lib)
            tmp = out + f".tmp{os.getpid()}"
            if LIBS[lib].get("torch", False):
                cmd = [CXX, "-o", tmp] + objs + _torch_flags()[1]
            else:
                cmd = [NVCC] + ARCH + ["-shared", "-Xcompiler", "-fopenmp", "-o", tmp] + objs
            _run(cmd, f"link of {lib}")
            os.replace(tmp, out)
            if LIBS[lib].get("torch", False):
                with open(out + ".tag", "w") as f:
                    f.write(_torch_tag())
    return {lib: os.path.join(OUT, lib) for lib in names}


if __name__ == "__main__":
    for name, path in build(force="--force" in sys.argv, quiet=False).items():
        print(name, path)
