"""Build the CUDA library ``libloomattn.so`` in-tree for sm_103a (GB300).

Each translation unit is compiled by nvcc in parallel, then linked into one shared
library next to this file.  No CMake, no torch extension machinery.  Beside it
``_binding.so``, the short way from Python to the entry points around training and serving
(it looks at tensors through torch's C++ interface; where the interpreter's or torch's headers
are missing, or it does not compile with them, it is left out, and the package's Python code does the same).
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libloomattn.so")
BINDING = os.path.join(HERE, "_binding.so")
SOURCES = ["loom_api.cu", "attn_fwd.cu", "attn_decode.cu", "loom_noalloc.cu", "gemm.cu",
           "attn_bwd.cu", "qkv_rope.cu", "attn_chunk.cu", "paged_plan.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "--expt-relaxed-constexpr",
                "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall"]


def _nvcc() -> str:
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    cand = os.path.join(cuda, "bin", "nvcc")
    return cand if os.path.exists(cand) else (shutil.which("nvcc") or "nvcc")


def _headers():
    hs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    hs.append(os.path.join(os.path.dirname(HERE), "include", "loom_attn.h"))
    return hs


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _binding_job(force: bool):
    """The command that compiles the binding, and the file it writes; None where there is nothing to do."""
    src, python = os.path.join(CSRC, "binding.cpp"), sysconfig.get_paths()["include"]
    spec = importlib.util.find_spec("torch")
    torch = os.path.dirname(spec.origin) if spec and spec.origin else ""
    needs = [os.path.join(python, "Python.h"), os.path.join(torch, "include", "torch", "csrc", "autograd", "python_variable.h"),
             os.path.join(torch, "lib", "libtorch_python.so")]
    deps = [src, os.path.join(os.path.dirname(HERE), "include", "loom_attn.h"), os.path.join(torch, "version.py")]
    if not all(map(os.path.exists, needs)) or not (force or _stale(BINDING, deps)):
        return None
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    tmp = BINDING + f".tmp{os.getpid()}"
    return ["g++", "-O2", "-std=c++17", "-Wall", "-fPIC", "-shared", f"-I{python}", "-isystem", os.path.join(torch, "include"),
            "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
            "-isystem", os.path.join(cuda, "include"), src, "-o", tmp, f"-L{os.path.join(torch, 'lib')}",
            "-ltorch_python", "-ltorch_cuda", "-lc10_cuda", "-ltorch_cpu", "-lc10"], tmp


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    """Compile (if needed) and return the path of ``libloomattn.so``."""
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    headers = _headers()
    objs = []
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + headers):
            extra = ["-Xptxas", "-v"] if ptxas_info else []
            jobs.append([nvcc, *FLAGS, *extra, "-c", s, "-o", o])

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"{os.path.basename(cmd[0])} failed ({' '.join(cmd)}):\n{r.stdout}\n{r.stderr}")
        if verbose or ptxas_info:
            print(r.stdout + r.stderr)

    def run_binding(cmd, made):
        try:
            run(cmd)
        except (OSError, RuntimeError) as e:
            if os.path.exists(BINDING):  # of another source or torch
                os.remove(BINDING)
            print(f"_binding.so is left out, the Python code takes its place: {e}", file=sys.stderr)
        else:
            os.replace(made, BINDING)

    binding = _binding_job(force)
    if jobs or binding:
        with ThreadPoolExecutor(max_workers=len(jobs) + 1) as ex:
            optional = ex.submit(run_binding, *binding) if binding else None
            list(ex.map(run, jobs))
            if optional:
                optional.result()
    if force or _stale(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        run([nvcc, *ARCH, "-shared", "-o", tmp, *objs])
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True, ptxas_info="--ptxas" in sys.argv))
