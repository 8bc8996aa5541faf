"""Builds libgreedylore.so (the C-ABI HIP library) for gfx950 in-tree.

    python -m paper_2507_08784_amd.build        # or build() from Python

Every .hip source under csrc/ is compiled with hipcc for gfx950 and linked
into paper_2507_08784_amd/libgreedylore.so next to this file; the Python
binding of the losses (csrc/losses_binding.cpp, host code on torch's C++
interface) is compiled with the host compiler into _losses.so beside it.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB_NAME = "libgreedylore.so"
BINDING_NAME = "_losses.so"
OBJ_DIR = os.path.join(HERE, "_build")

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-Wall",
    "-Wno-unused-function",
    # gfx950: keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE,
    "-I", CSRC,
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the GreedyLore HIP library cannot be built")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".hip"))


def _compile(src: str) -> str:
    obj = os.path.join(OBJ_DIR, os.path.basename(src) + ".o")
    cmd = [hipcc()] + HIPCC_FLAGS + ["-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    msg = "\n".join(l for l in (res.stdout + res.stderr).splitlines()
                    if "packed-fp32-ops" not in l and l.strip())
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {os.path.basename(src)}:\n{msg}")
    if msg:
        print(msg, file=sys.stderr)
    return obj


def _compile_binding() -> str:
    import torch
    from torch.utils.cpp_extension import include_paths

    src = os.path.join(CSRC, "losses_binding.cpp")
    obj = os.path.join(OBJ_DIR, "losses_binding.cpp.o")
    cmd = [os.environ.get("CXX") or shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", sysconfig.get_paths()["include"]]
    for p in include_paths():
        cmd += ["-isystem", p]
    res = subprocess.run(cmd + ["-c", src, "-o", obj], capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"compiling {os.path.basename(src)} failed:\n{res.stdout}{res.stderr}")
    return obj


def _link_binding(obj: str) -> None:
    import torch

    out = os.path.join(HERE, BINDING_NAME)
    cmd = [os.environ.get("CXX") or shutil.which("g++") or "c++", "-shared", "-fPIC", "-o", out + ".tmp", obj,
           "-L", os.path.join(os.path.dirname(torch.__file__), "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10",
           os.path.join(HERE, LIB_NAME), "-Wl,-rpath,$ORIGIN"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"linking {BINDING_NAME} failed:\n{res.stdout}{res.stderr}")
    os.replace(out + ".tmp", out)


def build(verbose: bool = True) -> str:
    """Compiles every source and links the shared library and the losses'
    binding; returns the library's path."""
    os.makedirs(OBJ_DIR, exist_ok=True)
    srcs = sources()
    with ThreadPoolExecutor(max_workers=8) as ex:
        binding = ex.submit(_compile_binding)
        objs = list(ex.map(_compile, srcs))
        binding = binding.result()
    out = os.path.join(HERE, LIB_NAME)
    tmp = out + ".tmp"
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", f"-Wl,-soname,{LIB_NAME}", "-o", tmp] + objs
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}{res.stderr}")
    os.replace(tmp, out)
    _link_binding(binding)
    if verbose:
        print(f"built {out}")
    return out


if __name__ == "__main__":
    build()
