"""Build libwino.so in-tree for gfx950 with hipcc.

Usage: python -m paper_1903_01521_amd.build [--check]
"""
from __future__ import annotations

import os
import re
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libwino.so")
KERNELS = [os.path.join(CSRC, f) for f in ("wino_kernels.hip", "wino_bf3.hip", "wino_bf3_1d.hip", "wino_gemm3.hip",
                                          "wino_norm.hip", "wino_wgrad.hip")]
SOURCES = KERNELS + [os.path.join(CSRC, f) for f in ("wino_api.cpp", "wino_train_api.cpp")]
HEADERS = [os.path.join(CSRC, f) for f in ("wino_device.h", "wino_transforms.h", "wino_internal.h", "wino_checks.h",
                                           "wino_fastdiv.h", "wino_norm.h", "wino_norm_device.h", "wino_wgrad.h")] + [
    os.path.join(ROOT, "include", "wino.h")]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
# Packed fp32 VALU ops are kept out of every kernel: plain fp32 FMA/add/mul only.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-I", os.path.join(ROOT, "include")]


def _each(f, items):
    """f of every item, several compilers at a time."""
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        return list(pool.map(f, items))


def build(verbose: bool = False) -> str:
    """Compile every HIP source into libwino.so (always recompiles)."""
    tmp = LIB + ".tmp%d" % os.getpid()
    with tempfile.TemporaryDirectory() as work:
        def compile_one(src):
            obj = os.path.join(work, os.path.basename(src) + ".o")
            cmd = [HIPCC] + COMMON + DEVICE_FLAGS + ["-c", "-o", obj, src]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.check_call(cmd)
            return obj
        objects = _each(compile_one, SOURCES)
        subprocess.check_call([HIPCC, "--offload-arch=" + ARCH, "-shared", "-o", tmp] + objects)
    os.replace(tmp, LIB)
    return LIB


def device_asm() -> str:
    """gfx950 assembly of the kernels (for inspection and the packed-op check)."""
    cmd = [HIPCC] + COMMON + DEVICE_FLAGS + ["--cuda-device-only", "-S", "-o", "-"]
    return "".join(_each(lambda k: subprocess.check_output(cmd + [k], text=True), KERNELS))


def resource_usage() -> str:
    """Per-kernel VGPR/AGPR/spill/occupancy report from the compiler."""
    cmd = [HIPCC] + COMMON + DEVICE_FLAGS + ["--cuda-device-only", "-c", "-o", os.devnull,
                                             "-Rpass-analysis=kernel-resource-usage"]
    return "".join(_each(lambda k: subprocess.run(cmd + [k], capture_output=True, text=True, check=True).stderr,
                         KERNELS))


def check_no_packed_fp32(asm: str | None = None) -> None:
    asm = device_asm() if asm is None else asm
    bad = re.findall(r"\bv_pk_(?:fma|mul|add)_f32\b", asm)
    if bad:
        raise RuntimeError(f"packed fp32 instructions in device code: {sorted(set(bad))}")


if __name__ == "__main__":
    print(build(verbose=True))
    if "--check" in sys.argv:
        check_no_packed_fp32()
        print(resource_usage())
