"""Compile librlattn.so (HIP for gfx950, with hipcc) and the binding's _pack.so (with g++) in-tree.

Usage: ``python -m paper_2609_08368_amd.build`` (``__graft_entry__.build()`` calls it).
"""

from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "librlattn.so")
PACK = os.path.join(PKG, "_pack.so")
ARCH = os.environ.get("RL_ATTN_ARCH", "gfx950")

SOURCES = ["decode.hip", "extend.hip", "append.hip", "map.hip", "requests.hip", "rope.hip", "rope_grad.hip", "prefill.hip",
           "logprob.hip", "diag.hip", "scratch.hip", "rl_attn_host.cpp"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build librlattn.so)")


def compiler() -> list:
    """hipcc with every option that decides the device code."""
    return [
        hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17",
        # packed FP32 instructions stay off: ordinary float code only
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        # device code: scores are never NaN unless the inputs are (a NaN still
        # reaches the output through the exponent), so fmaxf needs no NaN-quieting
        # canonicalisation; the host code keeps full NaN semantics
        "-Xarch_device", "-fno-honor-nans",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    ]


def build(verbose: bool = False) -> str:
    """Compile every HIP source into librlattn.so next to this file; returns its path."""
    out_tmp = LIB + ".tmp"
    cmd = [*compiler(), "-fPIC", "-shared", "-Wall", "-Wno-unused-result", *[os.path.join(CSRC, s) for s in SOURCES],
           "-o", out_tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    msgs = "\n".join(l for l in (res.stdout + res.stderr).splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{msgs}")
    if verbose and msgs.strip():
        print(msgs, file=sys.stderr)
    os.replace(out_tmp, LIB)
    build_pack(verbose)
    return LIB


def build_pack(verbose: bool = False) -> str:
    """Compile the binding's marshalling module (host code only) next to this file; returns its path."""
    import torch
    from torch.utils.cpp_extension import include_paths

    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    out_tmp = PACK + ".tmp"
    cmd = [
        os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
        f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
        "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"],
        *[a for p in include_paths() for a in ("-isystem", p)],
        "-Wall", os.path.join(CSRC, "pack.cpp"),
        "-L", libs, f"-Wl,-rpath,{libs}", "-ltorch_python", "-ltorch_cpu", "-lc10",
        "-o", out_tmp,
    ]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed ({res.returncode}):\n{res.stdout}{res.stderr}")
    os.replace(out_tmp, PACK)
    return PACK


if __name__ == "__main__":
    print(build(verbose=True))
