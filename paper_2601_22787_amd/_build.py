"""Compile libeq.so in place: gfx950 HIP kernels plus the host C++ parts."""
from __future__ import annotations

import os
import subprocess

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libeq.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
HIPCC = os.path.join(ROCM, "bin", "hipcc")

# Device code: gfx950 only; packed fp32 instructions disabled.
HIP_FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fno-strict-aliasing",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", INCLUDE, "-I", CSRC]
HOST_FLAGS = ["-O3", "-std=c++17", "-fPIC", "-pthread", "-D__HIP_PLATFORM_AMD__",
              "-I", INCLUDE, "-I", CSRC, "-I", os.path.join(ROCM, "include")]


def _run(cmd):
    subprocess.run(cmd, check=True)


def build(verbose: bool = False) -> str:
    """Always recompiles; returns the path of libeq.so."""
    os.makedirs(BUILD, exist_ok=True)
    objs = []
    for src in ("eq_encode.cpp", "eq_rd.cpp", "eq_layer.cpp"):
        obj = os.path.join(BUILD, src + ".o")
        _run(["g++", *HOST_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    for src in ("eq_decode.hip", "eq_decode2.hip", "eq_gemm.hip", "eq_kv.hip",
                "eq_attn.hip"):
        obj = os.path.join(BUILD, src + ".o")
        _run([HIPCC, *HIP_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    tmp = LIB + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-pthread", *objs, "-o", tmp])
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB
