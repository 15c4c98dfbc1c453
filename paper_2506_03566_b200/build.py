"""Builds libposs.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _paged_calls (its paged calls over torch
tensors, a Python module of C++) beside it."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libposs.so")
CALLS = os.path.join(HERE, "_paged_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
CALLS_TORCH = os.path.join(HERE, "_build", "_paged_calls.torch")   # the torch that it was built with
SOURCES = ["kernels_basic.cu", "kernels_attention.cu", "kernels_attention_mma.cu", "kernels_tree.cu", "gemm_tc.cu", "attention_tc.cu", "poss_api.cu", "no_alloc.cu",
           "paged_pages.cu", "paged_attention.cu", "paged_attention_tc.cu", "beam_select.cu"]
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_version() -> str:
    import torch
    return f"{torch.__version__} C++11 ABI {int(torch.compiled_with_cxx11_abi())}"


def _calls_stale(deps) -> bool:
    """_paged_calls reaches into torch's C++ by layout: it is as old as its sources, or as the torch that it was built with."""
    try:
        with open(CALLS_TORCH) as f:
            built_with = f.read()
    except OSError:
        return True
    return built_with != _torch_version() or _stale(CALLS, deps)


def build(force: bool = False, verbose: bool = False) -> str:
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers += [os.path.join(HERE, "..", "include", f) for f in ("poss.h", "poss_debug.h", "poss_paged.h")]
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    srcs = [s for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]
    objs = []
    procs = []
    for s in srcs:
        src = os.path.join(CSRC, s)
        obj = os.path.join(objdir, s.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, [src] + headers):
            cmd = [_nvcc()] + FLAGS + ["-c", src, "-o", obj]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
            procs.append((s, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for s, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode:
            sys.stderr.write(out)
        if p.returncode:
            raise RuntimeError(f"nvcc failed on {s}")
    if force or procs or _stale(OUT, objs):
        cmd = [_nvcc(), "-shared", "-o", OUT] + objs + ["-cudart", "static"]
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if r.returncode:
            sys.stderr.write(r.stdout)
            raise RuntimeError("link failed")
    src = os.path.join(CSRC, "paged_calls.cpp")
    if force or _calls_stale([src] + headers):
        import torch
        root = os.path.dirname(torch.__file__)
        cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(_nvcc()) or "/usr/local/cuda/bin/nvcc")))
        cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-shared",
               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
               f'-DPOSS_BUILT_WITH_TORCH="{_torch_version()}"', "-I" + sysconfig.get_paths()["include"],
               "-isystem", os.path.join(root, "include"),
               "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
               "-isystem", os.path.join(cuda, "include"), src, "-o", CALLS, "-L" + HERE, "-l:" + os.path.basename(OUT),
               "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
               "-l:libstdc++.so.6",    # torch's own: a second copy linked in would have locales of its own
               "-Wl,-rpath,$ORIGIN"]
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if r.returncode:
            sys.stderr.write(r.stdout)
            raise RuntimeError("g++ failed on paged_calls.cpp")
        with open(CALLS_TORCH, "w") as f:
            f.write(_torch_version())
    return OUT


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
