"""Builds libsds.so (the CUDA kernels and their C ABI) in-tree with nvcc for sm_100a, and the torch extension (the layer
operators on torch tensors, host code only) with the C++ compiler. The library does not need the extension."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsds.so")
EXT_SRC = os.path.join(CSRC, "sds_torch.cpp")

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
]


def sources() -> list:
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _older(built: str, deps: list) -> bool:
    return not os.path.exists(built) or any(os.path.getmtime(p) > os.path.getmtime(built) for p in deps)


def needs_build() -> bool:
    """Whether libsds.so is missing or older than what it is made of."""
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")]
    return _older(LIB, deps + [os.path.join(HERE, "..", "include", "sds.h")])


def ext_path() -> str:
    """The torch extension's file, one per version of torch and of Python (it is compiled against their headers)."""
    import sysconfig
    import torch
    return os.path.join(HERE, f"_sds_torch-{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}")


def needs_ext_build() -> bool:
    return _older(ext_path(), [EXT_SRC, os.path.join(HERE, "..", "include", "sds.h")])


def build(force: bool = False, verbose: bool = False) -> str:
    """Build what is older than its sources, or with `force` everything: libsds.so, then the torch extension. Returns the
    library path."""
    if force or needs_build():
        build_lib(force, verbose)
    if force or needs_ext_build():
        build_ext()
    return LIB


def build_lib(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ (one nvcc process per file, side by side) and link libsds.so. Objects go to _build/
    next to this file and are rebuilt only when a source or header is newer."""
    from concurrent.futures import ThreadPoolExecutor
    nvcc = os.environ.get("NVCC", "nvcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith((".cu", ".cpp"))]
    headers.append(os.path.join(HERE, "..", "include", "sds.h"))
    newest_header = max(os.path.getmtime(h) for h in headers)
    compile_flags = [f for f in NVCC_FLAGS if f != "-shared"]

    def compile_one(src: str):
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        if not force and os.path.exists(obj) and os.path.getmtime(obj) > max(os.path.getmtime(src), newest_header):
            return obj, None
        cmd = [nvcc] + compile_flags + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj, src]
        return obj, subprocess.run(cmd, capture_output=True, text=True)

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        results = list(pool.map(compile_one, sources()))
    for obj, res in results:
        if res is not None and res.returncode != 0:
            raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
        if res is not None and verbose:
            sys.stderr.write(res.stderr)
    res = subprocess.run([nvcc] + NVCC_FLAGS + ["-o", LIB] + [o for o, _ in results], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc link failed:\n" + res.stdout + res.stderr)
    return LIB


def build_ext() -> str:
    """Compile and link the torch extension against torch and the libsds.so next to it; returns its path."""
    import sysconfig
    import torch
    from torch.utils import cpp_extension
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    include = cpp_extension.include_paths() + [sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    ext = ext_path()
    tmp = f"{ext}.{os.getpid()}.tmp"                # (several processes may build at once: each puts a whole file in place)
    cmd = ([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"] + ["-isystem" + i for i in include]
           + [EXT_SRC, "-o", tmp, "-L" + torch_lib, "-L" + HERE, "-l:libsds.so", "-ltorch_python", "-ltorch_cpu",
              "-ltorch_cuda", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + torch_lib])
    try:
        res = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError(f"building the torch extension failed: {e}") from e
    if res.returncode != 0:
        raise RuntimeError("building the torch extension failed:\n" + res.stdout + res.stderr)
    os.replace(tmp, ext)
    return ext


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
