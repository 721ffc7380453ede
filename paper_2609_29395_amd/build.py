"""Build libgcpsl.so (HIP, gfx950) and _ops.so (its short way from Python) in-tree.

Usage: python -m paper_2609_29395_amd.build   (or build() from Python)
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJDIR = os.path.join(os.path.dirname(HERE), "_build", "gcpsl")
LIB = os.path.join(HERE, "libgcpsl.so")
BIND = os.path.join(HERE, "_ops.so")
SOURCES = ["api.cpp", "assign.cpp", "k_conv.hip", "k_conv_f32.hip", "k_misc.hip", "k_wgrad_lds.hip", "k_conv_lds.hip", "k_conv_img.hip", "k_norm.hip", "k_block.hip",
           "ops.cpp", "k_group.hip", "k_group_tile.hip", "k_group_f32.hip", "k_group_f32_deep.hip",
           "k_group_mid.hip",
           "k_group_few.hip", "k_score.hip", "k_drop.hip", "k_residual.hip", "k_distill.hip"]
ARCH = "gfx950"
FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17", "-Wall", "-Wshadow", "-Wno-unused-function",
    # keep the compiler from emitting packed fp32 arithmetic
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _hipcc() -> str:
    for c in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def _compile(src: str) -> str:
    obj = os.path.join(OBJDIR, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc(), "-x", "hip", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
    # report compiler warnings (the host pass's note about the gfx-only
    # packed-fp32 feature flag is expected)
    warn = [ln for ln in r.stderr.splitlines() if "warning:" in ln and "packed-fp32-ops" not in ln
            and "unused during compilation" not in ln]
    if warn:
        print(f"{src}:\n" + "\n".join(warn), file=sys.stderr)
    return obj


def _compile_bind() -> None:
    """csrc/bind.cpp against torch's headers: host code only."""
    import torch
    root = os.path.dirname(torch.__file__)
    include = os.path.join(root, "include")
    tmp = BIND + ".tmp"
    cmd = [_hipcc(), "-x", "c++", "-O2", "-fPIC", "-std=c++17", "-Wall", "-shared",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-isystem", include, "-isystem", os.path.join(include, "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "bind.cpp"), "-o", tmp,
           "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for bind.cpp:\n{r.stderr}")
    os.replace(tmp, BIND)


def build(verbose: bool = False) -> str:
    """Compile every HIP/C++ source for gfx950 and link libgcpsl.so and _ops.so."""
    os.makedirs(OBJDIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(6, len(SOURCES))) as ex:
        bind = ex.submit(_compile_bind)
        objs = list(ex.map(_compile, SOURCES))
        bind.result()
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
