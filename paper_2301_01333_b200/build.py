"""In-tree build of the CUDA library (sm_100a only) with nvcc.

``python -m paper_2301_01333_b200.build`` compiles ``csrc/*.cu`` into ``libgc_b200.so`` next to this
file, and ``csrc/serving_torch.cpp``, the torch side of ``serving.py``, into ``_serving.so``.  nvcc cross-compiles without a GPU,
so this also runs on a CPU-only box.  The C interface needs nothing but nvcc: where torch, its headers, Python's or a C++20 g++
are missing, the torch side is left out, with a line that says so, and only ``serving.py`` cannot be imported.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgc_b200.so")
TORCH_LIB = os.path.join(HERE, "_serving.so")
TORCH_SOURCE = os.path.join(CSRC, "serving_torch.cpp")
SOURCES = ["gc_api.cu", "gc_noalloc.cu", "kernels_generic.cu", "kernels_gemm_tc.cu", "kernels_gemm_tc2.cu", "kernels_chain.cu", "kernels_chain_cluster.cu",
           "kernels_sdpa_tc.cu", "kernels_sdpa_wide.cu", "kernels_sdpa_long.cu", "kernels_sdpa_small.cu",
           "gc_serving.cu", "kernels_qk_norm_rope.cu", "kernels_kv4.cu", "kernels_attn_kv4.cu", "kernels_attn_prompt.cu",
           "kernels_attn_chunk.cu", "kernels_kv4_weigh.cu", "kernels_kv4_evict.cu"]
HEADERS = ["gc_internal.h", "ptx.cuh", "epilogue.cuh", "gemm_epilogue.cuh", "serving.cuh", "attn_tc.cuh", os.path.join("..", "..", "include", "gc.h")]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS]
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_abi() -> str:
    """The torch and the Python that the torch side is compiled for; stands in ``_serving.so`` as a text."""
    import importlib.metadata
    import sysconfig
    try:
        version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        version = "none"
    return f"built for torch {version}, {sysconfig.get_config_var('SOABI')}"


def _torch_stale() -> bool:
    deps = [TORCH_SOURCE, os.path.join(HERE, "..", "include", "gc.h")]
    if not os.path.exists(TORCH_LIB) or any(os.path.getmtime(d) > os.path.getmtime(TORCH_LIB) for d in deps):
        return True
    with open(TORCH_LIB, "rb") as f:
        return _torch_abi().encode() + b"\0" not in f.read()


def _torch_side_lacks() -> str:
    """What the torch side cannot be compiled without and is not there, or an empty string."""
    import sysconfig
    try:
        import torch
        from torch.utils import cpp_extension as X
    except ImportError as e:
        return f"torch ({e})"
    if not any(os.path.exists(os.path.join(d, "ATen", "core", "Tensor.h")) for d in X.include_paths()):
        return f"the headers of torch {torch.__version__}"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    if not shutil.which("g++") or subprocess.run(["g++", "-std=c++20", "-fsyntax-only", "-x", "c++", os.devnull], capture_output=True).returncode:
        return "a g++ that knows C++20"
    return ""


def _torch_command():
    """The command that compiles ``_serving.so`` against the installed torch and the library next to it."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension as X
    inc = X.include_paths() + [sysconfig.get_paths()["include"], "/usr/local/cuda/include"]
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    return (["g++", "-O2", "-std=c++20", "-fPIC", "-shared", "-fvisibility=hidden",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DSERVING_ABI="{_torch_abi()}"']
            + [a for d in inc for a in ("-isystem", d)] + [TORCH_SOURCE, "-o", TORCH_LIB + ".new", LIB, "-L" + libs]
            + ["-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN"])


def _build_torch(verbose: bool) -> None:
    r = subprocess.run(_torch_command(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or r.returncode != 0:
        sys.stderr.write(r.stdout)
    if r.returncode != 0:
        raise RuntimeError("g++ failed on serving_torch.cpp")
    os.replace(TORCH_LIB + ".new", TORCH_LIB)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile what is missing or older than its sources; return the path of the CUDA library."""
    if force or _stale():
        _build_cuda(verbose)
    if force or _torch_stale():
        lacks = _torch_side_lacks()
        if lacks:
            sys.stderr.write(f"serving.py's torch side is left out: {lacks} is missing\n")
        else:
            _build_torch(verbose)
    return LIB


def _build_cuda(verbose: bool) -> None:
    nvcc = _nvcc()
    objs = []
    bdir = os.path.join(HERE, "build")
    os.makedirs(bdir, exist_ok=True)
    procs = []
    for s in SOURCES:
        o = os.path.join(bdir, s.replace(".cu", ".o"))
        objs.append(o)
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", os.path.join(CSRC, s), "-o", o]
        procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for s, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError(f"nvcc failed on {s}")
    cmd = [nvcc, "-shared", "-o", LIB, "-Xlinker", "-soname=libgc_b200.so"] + objs + ["-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static"]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout)
        raise RuntimeError("link failed")


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
