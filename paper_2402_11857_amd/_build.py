"""Compiles the HIP library for gfx950 in-tree (paper_2402_11857_amd/libliec.so)."""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
LIB_PATH = os.path.join(_HERE, "libliec.so")
SOURCES = [os.path.join(_HERE, "csrc", n) for n in ("liec_api.hip", "train_api.hip", "activations_api.hip")]
HEADERS = [os.path.join(_HERE, "csrc", n) for n in ("liec_kernels.hpp", "operands.hpp", "spans.hpp")] + \
          [os.path.join(_ROOT, "include", n) for n in ("liec.h", "liec_testing.h", "liec_train.h", "liec_activations.h")] + \
          [os.path.join(_HERE, "csrc", "kernels", n)
           for n in ("checkpoint.hpp", "common.hpp", "elements.hpp", "grads.hpp", "group_norm.hpp", "group_norm_held.hpp", "layer_norm.hpp", "rows.hpp", "select.hpp", "sign.hpp",
                     "step.hpp", "sync.hpp", "telemetry.hpp", "weight_grad.hpp", "wire.hpp")]


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the HIP library cannot be built")


def build_library(verbose: bool = False, defines=(), out: str = LIB_PATH) -> str:
    """Always recompiles.  -ffp-contract=off keeps every fp32 expression a single IEEE operation;
    packed fp32 instructions are disabled for the device pass.  A kernel's leading arguments, up to 14 words of them and none from
    the first struct passed by value on, are in scalar registers when a wave starts instead of being loaded by every wave (short
    kernels gain most: 8 scaled-sign messages of 11.7M + 1 columns 101.7 -> 98.9 us, averaging 27 x 109160 13.6 -> 13.0, top-k
    8 x 1M 53.2 -> 52.2; long ones are even).  `defines` (NAME=value strings) and `out`
    let a tuning run build a variant of the library beside the product's.  The sources are compiled side by side."""
    flags = [hipcc(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
             "-ffp-contract=off", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-mllvm", "-amdgpu-kernarg-preload-count=16",
             "-Wall", "-Wno-unused-command-line-argument"] + [f"-D{d}" for d in defines] + [
             "-I", os.path.join(_ROOT, "include"), "-I", os.path.join(_HERE, "csrc")]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
        if verbose and res.stderr.strip():
            print(res.stderr)

    with tempfile.TemporaryDirectory() as tmp, concurrent.futures.ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        list(pool.map(lambda pair: run(flags + ["-c", pair[0], "-o", pair[1]]), zip(SOURCES, objects)))
        run([hipcc(), "--offload-arch=gfx950", "-fPIC", "-shared", "-o", out] + objects)
    return out


BINDING_PATH = os.path.join(_HERE, "_train.so")


def host_compiler() -> str:
    """A C++ compiler for host code: the system's, or the one that comes with hipcc."""
    for cand in (shutil.which("g++"), shutil.which("c++"), os.path.join(os.path.dirname(hipcc()), "amdclang++")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("no C++ compiler found: the binding cannot be built")


def build_binding(verbose: bool = False) -> str:
    """Always recompiles the Python side of include/liec_train.h and include/liec_activations.h (host code only, against the headers
    of Python and torch).  The compressed step does not need it."""
    import sysconfig

    from torch.utils import cpp_extension

    python = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(python, "Python.h")):
        raise RuntimeError(f"{os.path.join(python, 'Python.h')} not found: the binding cannot be built without Python's headers")
    cmd = [host_compiler(), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-I", os.path.join(_ROOT, "include")]
    for path in cpp_extension.include_paths() + [python]:
        cmd += ["-isystem", path]
    cmd += [os.path.join(_HERE, "csrc", n) for n in ("train_binding.cpp", "activations_binding.cpp")] + ["-o", BINDING_PATH]
    for path in cpp_extension.library_paths():
        cmd += ["-L", path]
    cmd += ["-lc10", "-ltorch_cpu", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("the binding did not compile:\n" + res.stdout + res.stderr)
    return BINDING_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_binding(verbose=True))
