"""Build libpatconv.so in-tree: nvcc for the sm_103a kernels, g++ for the host packer; and beside it, where torch
is installed, _patconv.so, the native binding of the training side, which links against torch and the library.

Both are written to ``paper_2003_06513_gb300/_build/`` (git-ignored), and each is rebuilt whenever a source
file or a flag of its own changes, the binding with the torch version too.  No CMake: nine translation units compiled in parallel and
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
from typing import Optional

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
SOURCES = KERNELS + ["tensor.h", "norm.h", "norm.cuh", "pack.cpp", "layer.h", "gen_dispatch.py"]


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


def _digest(sources, *more) -> str:
    h = hashlib.sha256()
    for name in sources + [os.path.join("..", "..", "include", "patconv.h")]:
        with open(os.path.join(CSRC, name), "rb") as f:
            h.update(f.read())
    h.update(repr(more).encode())
    return h.hexdigest()


def _obj(name: str) -> str:
    return os.path.join(BUILD, name.split(".")[0] + ".o")


class _Part:
    """One of the two products: compiled where it, or the digest of what it is made of, is not there."""

    def __init__(self, path: str, stamp: str, digest: str, force: bool):
        self.path, self.stamp, self.digest = path, os.path.join(BUILD, stamp), digest
        self.stale = force or not all(os.path.exists(f) for f in (path, self.stamp))
        if not self.stale:
            with open(self.stamp) as f:
                self.stale = f.read().strip() != digest

    def link(self, run, cmd) -> None:
        tmp = self.path + ".tmp"
        run([tmp if c is None else c for c in cmd])
        os.replace(tmp, self.path)
        with open(self.stamp, "w") as f:
            f.write(self.digest)


def build(force: bool = False, verbose: bool = False, extra_nvcc=(), binding: Optional[bool] = None) -> str:
    """Compile what is stale and return the path of libpatconv.so.  The library needs nvcc and g++ alone.  ``binding``:
    whether _patconv.so is built beside it; None: where torch is installed; True raises RuntimeError without it."""
    os.makedirs(BUILD, exist_ok=True)
    if binding is None:
        binding = importlib.util.find_spec("torch") is not None
    library = _Part(LIB, "stamp", _digest(SOURCES, NVCC_FLAGS, GXX_FLAGS, tuple(extra_nvcc)), force)
    parts = [library]
    if binding:
        torch_dir = _torch_dir()
        parts.append(_Part(BINDING, "stamp_binding", _digest(["binding.cpp"], GXX_FLAGS, _torch_version(torch_dir)), force))
    if not any(p.stale for p in parts):
        return LIB
    nvcc = _nvcc()

    def run(cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0 or verbose:
            sys.stderr.write(" ".join(cmd) + "\n" + r.stdout + r.stderr)
        if r.returncode != 0:
            raise RuntimeError(f"build step failed: {' '.join(cmd[:3])}")
        return r.stdout + r.stderr

    with ThreadPoolExecutor(max_workers=len(KERNELS) + 2) as ex:
        glue = None
        if binding and parts[1].stale:
            cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))
            includes = [os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
                        os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
            glue = ex.submit(run, ["g++", "-c", os.path.join(CSRC, "binding.cpp"), "-o", _obj("binding.cpp")] + GXX_FLAGS
                             + [f for d in includes for f in ("-isystem", d)])
        if library.stale:
            run([sys.executable, os.path.join(CSRC, "gen_dispatch.py"), os.path.join(BUILD, "pattern_dispatch.h")])
            cmds = [[nvcc, "-c", os.path.join(CSRC, name), "-o", _obj(name), "-I", BUILD] + NVCC_FLAGS + list(extra_nvcc)
                    for name in KERNELS]
            cmds += [["g++", "-c", os.path.join(CSRC, "pack.cpp"), "-o", _obj("pack.cpp")] + GXX_FLAGS]
            list(ex.map(run, cmds))
            library.link(run, [nvcc, "-shared", "-o", None] + [_obj(name) for name in KERNELS + ["pack.cpp"]] + ARCH
                         + ["-cudart", "static"])
        if glue is not None:
            glue.result()
            lib = os.path.join(torch_dir, "lib")
            parts[1].link(run, ["g++", "-shared", "-o", None, _obj("binding.cpp"), "-L", BUILD, "-l:libpatconv.so", "-L", lib, "-lc10",
                                "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN:" + lib])
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
