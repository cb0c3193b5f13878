"""Builds libmuloco.so (hand-written CUDA for sm_100a) in-tree with nvcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmuloco.so")
LIB_DEBUG = os.path.join(HERE, "libmuloco_debug.so")   # the same sources with -DMULOCO_DEBUG (index checks of the optimizer's kernels)
SOURCES = ["capi.cu", "elementwise.cu", "outer_sync.cu", "topk.cu", "ns_fp32.cu", "ns_tc.cu", "ns_static.cu",
           "adamw.cu", "qk_norm.cu", "ffn.cu", "ops_capi.cu"]


def _nvcc() -> str:
    cand = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: libmuloco cannot be built")
    return cand


def needs_build(lib_path: str = LIB) -> bool:
    if not os.path.exists(lib_path):
        return True
    t = os.path.getmtime(lib_path)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h"))]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "muloco.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False, lib_path: str = None, debug: bool = False) -> str:
    """Compile every CUDA source of the package for sm_100a into one shared library.
    debug=True builds libmuloco_debug.so: the same sources with -DMULOCO_DEBUG, i.e. with the
    index checks of the Newton-Schulz, sync and inner-step AdamW kernels compiled in (a failed check raises a status flag, nothing traps)."""
    if lib_path is None:
        lib_path = LIB_DEBUG if debug else LIB
    if lib_path == LIB:
        # the library needs neither g++ nor torch's headers, and the binding does without the call path
        try:
            build_fastcall()
        except Exception as e:                   # noqa: BLE001 - whatever keeps it from being built
            if os.path.exists(FASTCALL):
                os.remove(FASTCALL)              # made for other sources or another torch
            sys.stderr.write(f"_fastcall.so was not built ({e}): the operators' calls are marshalled in Python\n")
    if not force and lib_path in (LIB, LIB_DEBUG) and not needs_build(lib_path):
        return lib_path
    objs = []
    bdir = os.path.join(HERE, "_build") if lib_path == LIB else (
        os.path.join(HERE, "_build", "debug") if lib_path == LIB_DEBUG else lib_path + ".objs")
    os.makedirs(bdir, exist_ok=True)
    common = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden"]
    if debug:
        common += ["-DMULOCO_DEBUG"]
    if verbose:
        common += ["-Xptxas", "-v"]
    common += os.environ.get("MULOCO_NVCC_FLAGS", "").split()   # extra -D... for tuning studies
    procs = []
    for src in SOURCES:
        obj = os.path.join(bdir, src.replace(".cu", ".o"))
        objs.append(obj)
        procs.append((src, subprocess.Popen(common + ["-c", os.path.join(CSRC, src), "-o", obj],
                                            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    subprocess.check_call([_nvcc(), "-shared", "-o", lib_path] + objs)
    return lib_path


FASTCALL = os.path.join(HERE, "_fastcall.so")
FASTCALL_TORCH = os.path.join(HERE, "_build", "fastcall.torch")    # the torch version that it was made for


def build_fastcall(force: bool = False) -> str:
    """Compile the operators' call path (csrc/fastcall.cpp: a CPython module over torch's C++ interface, host code
    only) next to the library."""
    src = os.path.join(CSRC, "fastcall.cpp")
    deps = [src, os.path.join(os.path.dirname(HERE), "include", "muloco.h")]
    from importlib.metadata import version
    made_for = open(FASTCALL_TORCH).read() if os.path.exists(FASTCALL_TORCH) else None
    if not force and os.path.exists(FASTCALL) and made_for == version("torch") and \
            all(os.path.getmtime(FASTCALL) >= os.path.getmtime(d) for d in deps):
        return FASTCALL
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    lib = os.path.join(root, "lib")
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DMULOCO_TORCH="{torch.__version__}"',
           "-isystem", os.path.join(root, "include"), "-isystem", cuda, "-isystem", sysconfig.get_paths()["include"],
           src, "-o", FASTCALL, "-L" + lib, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath," + lib]
    p = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if p.returncode != 0:
        sys.stderr.write(p.stdout)
        raise RuntimeError("g++ failed on fastcall.cpp")
    os.makedirs(os.path.dirname(FASTCALL_TORCH), exist_ok=True)
    with open(FASTCALL_TORCH, "w") as f:
        f.write(version("torch"))
    return FASTCALL


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
    print(build_fastcall(force=True))
