"""Build libwsr_step.so (the operators of include/wsr_step.h, HIP kernels for gfx950 plus the C ABI) in-tree with
hipcc: the flags and the toolchain checks of build.py, in a library of its own so that libwsr.so, whose counters are
tied to its sources, stays as it is."""
from __future__ import annotations

import os

from . import build as wb

LIB_PATH = os.path.join(wb.PKG, "libwsr_step.so")
KERNEL_FILES = ("wsr_norm.hip", "wsr_lora.hip", "wsr_attn.hip", "wsr_verify.hip")


def _compile_api() -> str:
    obj = os.path.join(wb.OUT_DIR, "wsr_step_api.o")
    wb._run(["hipcc", *wb.COMMON, "-c", os.path.join(wb.CSRC, "wsr_step_api.cpp"), "-o", obj])
    return obj


def build(verbose: bool = False) -> str:
    """Compile the kernel files and the C ABI side by side, then link and move the library into place in
    one rename."""
    from concurrent.futures import ThreadPoolExecutor
    os.makedirs(wb.OUT_DIR, exist_ok=True)
    with ThreadPoolExecutor(len(KERNEL_FILES) + 1) as ex:
        futs = [ex.submit(wb._compile_kernels, src) for src in KERNEL_FILES]
        api = ex.submit(_compile_api)
        objs = [f.result() for f in futs] + [api.result()]
    tmp = LIB_PATH + ".tmp"
    wb._run(["hipcc", "-shared", "-fPIC", f"--offload-arch={wb.ARCH}", *objs, "-o", tmp])
    os.replace(tmp, LIB_PATH)
    if verbose:
        print("built", LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    build(verbose=True)
