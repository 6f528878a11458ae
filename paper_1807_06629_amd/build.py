"""Builds libprsgd.so (HIP, gfx950 only) in-tree with hipcc, and the Python module of its operators with g++.

    python -m paper_1807_06629_amd.build

Each translation unit under csrc/ is compiled to an object in _build/ and the objects are
linked into paper_1807_06629_amd/libprsgd.so; csrc/binding becomes paper_1807_06629_amd/_ops.so beside it.  Packed-FP32 instruction selection is turned off
for all device code.
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
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libprsgd.so")
BINDING = os.path.join(HERE, "_ops.so")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _hipcc() -> str:
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found")
    return exe


def _run(cmd):
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in proc.stdout.splitlines()
                    if "is not a recognized feature for this target" not in l)
    if proc.returncode != 0:
        raise RuntimeError("command failed: %s\n%s" % (" ".join(cmd), out))
    return out


def _build_binding() -> str:
    """Torch tensors to the operators' C calls: host code only, linked to the libprsgd.so beside it."""
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    return _run([shutil.which("g++") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
                 "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", "-I", os.path.join(ROOT, "include"),
                 "-I", sysconfig.get_paths()["include"], "-I", os.path.join(torch, "include"),
                 "-I", os.path.join(torch, "include", "torch", "csrc", "api", "include"), "-I", os.path.join(rocm, "include"),
                 os.path.join(CSRC, "binding", "ops_binding.cpp"), "-o", BINDING, "-L", os.path.join(torch, "lib"),
                 "-ltorch_python", "-ltorch_cpu", "-ltorch_hip", "-lc10", "-lc10_hip", "-L", HERE, "-l:libprsgd.so", "-Wl,-rpath,$ORIGIN"])


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    hipcc = _hipcc()
    sources = sorted(f for f in os.listdir(CSRC) if f.endswith(".hip"))
    objects = [os.path.join(BUILD, f[:-4] + ".o") for f in sources]

    def compile_one(pair):
        src, obj = pair
        return _run([hipcc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])

    with ThreadPoolExecutor(max_workers=min(8, len(sources))) as pool:
        for log in pool.map(compile_one, zip(sources, objects)):
            if verbose and log.strip():
                print(log)
    log = _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objects])
    if verbose and log.strip():
        print(log)
    log = _build_binding()
    if verbose and log.strip():
        print(log)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
