"""Build libpatconv.so in-tree: nvcc for the sm_103a kernels, g++ for the host packer; and beside it
_patconv.so, the native binding of the training side, which links against torch and the library.

Both are written to ``paper_2003_06513_gb300/_build/`` (git-ignored) and are rebuilt whenever a source
file, a flag or the torch version changes.  No CMake: nine translation units compiled in parallel and
two links, so a fresh build takes a minute or so, the largest unit's time.
"""
from __future__ import annotations

import hashlib
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(BUILD, "libpatconv.so")
BINDING = os.path.join(BUILD, "_patconv.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-lineinfo", "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC",
              "-Xcompiler", "-ffp-contract=off", "-I", os.path.join(ROOT, "include")] + ARCH
GXX_FLAGS = ["-O2", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Wall", "-I",
             os.path.join(ROOT, "include")]
KERNELS = ["conv.cu", "tensor.cu", "norm.cu", "norm_f32.cu", "norm_f16.cu", "norm_bf16.cu", "optim.cu"]
SOURCES = KERNELS + ["tensor.h", "norm.h", "norm.cuh", "pack.cpp", "layer.h", "gen_dispatch.py", "binding.cpp"]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libpatconv")


def _torch_dir() -> str:
    """torch's folder, without the time that importing it takes."""
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.submodule_search_locations:
        raise RuntimeError("torch not found: the package's binding is built against it")
    return spec.submodule_search_locations[0]


def _torch_version(torch_dir: str) -> str:
    with open(os.path.join(torch_dir, "version.py")) as f:
        return f.read()


def _digest(extra) -> str:
    h = hashlib.sha256(_torch_version(_torch_dir()).encode())
    for name in SOURCES + [os.path.join("..", "..", "include", "patconv.h")]:
        with open(os.path.join(CSRC, name), "rb") as f:
            h.update(f.read())
    h.update(repr((NVCC_FLAGS, GXX_FLAGS, extra)).encode())
    return h.hexdigest()


def build(force: bool = False, verbose: bool = False, extra_nvcc=()) -> str:
    """Compile (if stale) and return the path of libpatconv.so."""
    os.makedirs(BUILD, exist_ok=True)
    stamp = os.path.join(BUILD, "stamp")
    digest = _digest(tuple(extra_nvcc))
    if not force and all(os.path.exists(f) for f in (LIB, BINDING, stamp)):
        with open(stamp) as f:
            if f.read().strip() == digest:
                return LIB
    nvcc = _nvcc()
    subprocess.run([sys.executable, os.path.join(CSRC, "gen_dispatch.py"),
                    os.path.join(BUILD, "pattern_dispatch.h")], check=True)
    torch_dir = _torch_dir()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))
    includes = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
                os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]

    def obj(name):
        return os.path.join(BUILD, name.split(".")[0] + ".o")

    cmds = [[nvcc, "-c", os.path.join(CSRC, name), "-o", obj(name), "-I", BUILD] + NVCC_FLAGS + list(extra_nvcc)
            for name in KERNELS]
    cmds += [["g++", "-c", os.path.join(CSRC, "pack.cpp"), "-o", obj("pack.cpp")] + GXX_FLAGS,
             ["g++", "-c", os.path.join(CSRC, "binding.cpp"), "-o", obj("binding.cpp")] + GXX_FLAGS
             + [f for d in includes for f in ("-isystem", d)]]

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0 or verbose:
            sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"build step failed: {' '.join(cmd[:3])}")
        return r.stdout + r.stderr

    with ThreadPoolExecutor(max_workers=len(cmds)) as ex:
        list(ex.map(run, cmds))
    tmp = LIB + ".tmp"
    run([nvcc, "-shared", "-o", tmp] + [obj(name) for name in KERNELS + ["pack.cpp"]] + ARCH + ["-cudart", "static"])
    os.replace(tmp, LIB)
    tmp, lib = BINDING + ".tmp", os.path.join(torch_dir, "lib")
    run(["g++", "-shared", "-o", tmp, obj("binding.cpp"), "-L", BUILD, "-l:libpatconv.so", "-L", lib, "-lc10", "-lc10_cuda",
         "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN:" + lib])
    os.replace(tmp, BINDING)
    with open(stamp, "w") as f:
        f.write(digest)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
