"""Builds libs1f.so (HIP kernels + C ABI) in-tree with hipcc for gfx950."""
from __future__ import annotations

import os
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libs1f.so")
CALLS_LIB = os.path.join(HERE, "_torch_calls.so")   # the tensor calls of binding.py
PROBE_LIB = os.path.join(HERE, "libs1f_probe.so")   # measurement aid used by bench.py only

SOURCES = ["s1f_api.hip", "s1f_cache.hip", "s1f_embed.hip", "s1f_norm.hip", "s1f_loss.hip", "s1f_rope.hip", "s1f_ffn.hip", "s1f_partition.cpp", "s1f_schedule.cpp", "s1f_pipeline.cpp"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Werror=array-bounds",
         # packed fp32 VALU forms are kept out of generated code on this target
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _run(cmd) -> str:
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + proc.stdout + proc.stderr)
    return proc.stderr


def build_library(verbose: bool = False) -> str:
    """Sources side by side, as many as there are processors for (one after the other: 128 s), then the link."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    compile_flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1, 16)) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        said = list(pool.map(lambda s, o: _run([hipcc, *compile_flags, f"-I{INCLUDE}", f"-I{CSRC}", "-c", os.path.join(CSRC, s), "-o", o]), SOURCES, objects))
        said.append(_run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", LIB, *objects]))
    if verbose:
        print("".join(said))
    build_calls()
    _run([hipcc, *FLAGS, "-o", PROBE_LIB, os.path.join(CSRC, "mfma_peak.hip")])
    return LIB


def build_calls() -> None:
    """The extension module of the tensor calls: host code against torch's headers."""
    import torch
    root = os.path.dirname(torch.__file__)
    include, lib = os.path.join(root, "include"), os.path.join(root, "lib")
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f"-I{INCLUDE}", f"-isystem{include}",
           f"-isystem{os.path.join(include, 'torch', 'csrc', 'api', 'include')}", f"-isystem{sysconfig.get_paths()['include']}",
           os.path.join(CSRC, "torch_calls.cpp"), "-o", CALLS_LIB, f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10"]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("g++ failed:\n" + proc.stdout + proc.stderr)


if __name__ == "__main__":
    print(build_library(verbose=True))
