"""Build libblink.so (CUDA kernels + C ABI) in-tree for sm_100a with nvcc, and beside it, where there is torch, _marshal.so, which hands torch
tensors to it."""
from __future__ import annotations

import importlib.metadata
import importlib.util
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libblink.so")
OBJ = os.path.join(HERE, "_build")
MARSHAL = os.path.join(HERE, "_marshal.so")


def _newest(paths):
    return max(os.path.getmtime(p) for p in paths)


def sources():
    out = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith((".cu", ".cuh", ".h"))]
    out.append(os.path.join(os.path.dirname(HERE), "include", "blink.h"))
    return out


def marshal_for() -> str:
    """What _marshal.so is built for: this torch and this Python.  It says so in itself."""
    try:
        version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:   # (one that was not installed as a package)
        import torch
        version = torch.__version__
    return f"torch {version}, {sysconfig.get_config_var('SOABI')}"


def build_marshal(force: bool = False) -> str:
    """The operators' argument marshalling, against torch's headers (g++; no device code)."""
    src = os.path.join(CSRC, "marshal.cpp")
    if not force and os.path.exists(MARSHAL) and os.path.getmtime(MARSHAL) >= _newest([src, os.path.join(CSRC, "ops.h"), os.path.join(os.path.dirname(HERE), "include", "blink.h")]):
        with open(MARSHAL, "rb") as f:
            if f"built for {marshal_for()}.".encode() in f.read():
                return MARSHAL
    import torch
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DBLINK_BUILT_FOR="{marshal_for()}"']
    cmd += ["-isystem" + d for d in (os.path.join(home, "include"), os.path.join(cuda, "include"), sysconfig.get_paths()["include"])]
    cmd += [src, "-o", MARSHAL, "-L" + HERE, "-l:libblink.so", "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(home, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu",
            "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("g++ failed building _marshal.so")
    return MARSHAL


def build(force: bool = False, verbose: bool = False) -> str:
    lib = build_library(force, verbose)
    if importlib.util.find_spec("torch"):
        build_marshal(force)
    else:   # the library, and all of it but the operators' calls with tensors, does without
        sys.stderr.write("no torch: _marshal.so is not built\n")
    return lib


def build_library(force: bool = False, verbose: bool = False) -> str:
    srcs = sources()
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest(srcs):
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    os.makedirs(OBJ, exist_ok=True)
    units = [f for f in sorted(os.listdir(CSRC)) if f.endswith(".cu")]

    def compile_one(f):
        obj = os.path.join(OBJ, f[:-3] + ".o")
        r = subprocess.run([nvcc] + flags + ["-c", os.path.join(CSRC, f), "-o", obj], capture_output=True, text=True)
        return f, obj, r

    # one translation unit per kernel variant family, compiled side by side
    with ThreadPoolExecutor(max_workers=min(len(units), os.cpu_count() or 1)) as ex:
        results = list(ex.map(compile_one, units))
    log = ""
    for f, obj, r in results:
        log += f"==== {f}\n{r.stdout}{r.stderr}"
        if r.returncode != 0:
            sys.stderr.write(log)
            raise RuntimeError(f"nvcc failed compiling {f}")
    r = subprocess.run([nvcc, "-shared", "-o", LIB] + [obj for _, obj, _ in results], capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("nvcc failed linking libblink.so")
    if verbose:
        print(log)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
