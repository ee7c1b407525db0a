"""Build the HIP library ``libspec_verify.so`` for gfx950 in-tree with hipcc.

A kernel source is compiled in two passes so that each pass gets only the
flags meant for it: the device pass (``--cuda-device-only``) is built with
packed-fp32 instruction formation disabled, and its fat binary is embedded
into the host pass (``--cuda-host-only``).  Both passes and the host-only
decoding loop build with ``-Wall -Wextra -Werror``.  The sources are compiled
side by side.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_NAME = "libspec_verify.so"
LIB_PATH = os.path.join(PKG_DIR, LIB_NAME)
KERNEL_SOURCE = os.path.join(CSRC, "spec_verify.hip")
CACHE_SOURCES = [os.path.join(CSRC, name) for name in ("cache.hip", "cache_attend.hip", "cache_attend_f16.hip")]
KERNEL_SOURCES = [KERNEL_SOURCE, *CACHE_SOURCES]
HOST_SOURCES = [os.path.join(CSRC, "decode_loop.hip")]
SOURCES = [*KERNEL_SOURCES, *HOST_SOURCES]
ARCH = "gfx950"

COMMON_FLAGS = ["-O3", "-std=c++17", "-Wall", "-Wextra", "-Werror"]
# device code: no packed-fp32 instructions (the compiler would otherwise form
# them from scalar and float2 code)
DEVICE_FLAGS = [f"--offload-arch={ARCH}", "--cuda-device-only", "-munsafe-fp-atomics",
                "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
HOST_FLAGS = [f"--offload-arch={ARCH}", "--cuda-host-only", "-fPIC"]


def hipcc() -> str:
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found; the HIP library cannot be built")
    return path


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"hipcc failed with status {res.returncode}")
    if res.stderr.strip():
        # -Werror turns every diagnostic into a failure; anything printed
        # here is a note from a tool, shown as is
        sys.stderr.write(res.stderr)


def _compile_kernels(src: str, tmpdir: str, flags, verbose: bool) -> str:
    name = os.path.splitext(os.path.basename(src))[0]
    fatbin, obj = os.path.join(tmpdir, name + ".hipfb"), os.path.join(tmpdir, name + ".o")
    _run([hipcc(), *COMMON_FLAGS, *DEVICE_FLAGS, *flags, "-c", src, "-o", fatbin], verbose)
    _run([hipcc(), *COMMON_FLAGS, *HOST_FLAGS, *flags, "-Xclang", "-fcuda-include-gpubinary", "-Xclang", fatbin, "-c",
          src, "-o", obj], verbose)
    return obj


def _compile_host(src: str, tmpdir: str, flags, verbose: bool) -> str:
    obj = os.path.join(tmpdir, os.path.splitext(os.path.basename(src))[0] + ".o")
    _run([hipcc(), *COMMON_FLAGS, *HOST_FLAGS, *flags, "-c", src, "-o", obj], verbose)
    return obj


def build(verbose: bool = False, extra_flags=None) -> str:
    """Compile the library; returns its path.  Always recompiles."""
    flags = [*(extra_flags or []), "-I", INCLUDE, "-I", CSRC]
    with tempfile.TemporaryDirectory(prefix="sv_build_") as tmpdir, ThreadPoolExecutor(len(SOURCES)) as pool:
        jobs = [pool.submit(_compile_kernels, src, tmpdir, flags, verbose) for src in KERNEL_SOURCES]
        jobs += [pool.submit(_compile_host, src, tmpdir, flags, verbose) for src in HOST_SOURCES]
        objs = [j.result() for j in jobs]
        tmp = LIB_PATH + ".tmp"
        _run([hipcc(), "-shared", "-fPIC", *objs, "-o", tmp], verbose)
        os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
