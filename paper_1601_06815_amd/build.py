"""Build liboaa.so (the C-ABI library of include/oaa.h) for gfx950 with hipcc.

Every HIP source is compiled for gfx950 only, with packed-fp32 instructions
disabled; objects go to ``_build/`` next to this file and the shared library
to ``liboaa.so`` in the package directory, where the binding loads it.
"""

import concurrent.futures
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(HERE, "_build")
LIB_PATH = os.path.join(HERE, "liboaa.so")
SOURCES = ["oaa_plan.cpp", "k_tile_fft.hip", "k_fold_fft.hip", "k_big_fft.hip", "k_wide_fft.hip", "k_fused.hip", "k_cgemm.hip", "k_narrow.hip",
           "oaa_norm.cpp", "k_norm_planes_f32.hip", "k_norm_planes_bf16.hip", "k_norm_planes_f16.hip", "k_norm_last_f32.hip",
           "k_norm_last_bf16.hip", "k_norm_last_f16.hip", "k_group_norm.hip", "oaa_grad.cpp", "k_grad.hip"]

HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(src, build_dir=BUILD_DIR, defines=()):
    obj = os.path.join(build_dir, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *[f"-D{d}" for d in defines], "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose=False, lib_path=LIB_PATH, build_dir=BUILD_DIR, defines=()):
    """Compile all sources and link liboaa.so; returns the library path.
    ``defines`` are extra NAME=VALUE preprocessor definitions (launch-shape
    overrides for tuning builds)."""
    os.makedirs(build_dir, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, build_dir, defines), SOURCES))
    tmp = lib_path + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib_path)
    if verbose:
        print(f"built {lib_path}")
    return lib_path


if __name__ == "__main__":
    build(verbose=True)
