"""Build libwsr_serve.so (the operators of include/wsr_serve.h, HIP kernels for gfx950 plus the C ABI) in-tree with
hipcc: the flags and the toolchain checks of build.py, in a library of its own like libwsr_step.so."""
from __future__ import annotations

import os

from . import build as wb

LIB_PATH = os.path.join(wb.PKG, "libwsr_serve.so")
KERNEL_FILES = ("wsr_append.hip", "wsr_paged.hip", "wsr_paged_rows.hip", "wsr_logprobs.hip")


def _compile_api() -> str:
    obj = os.path.join(wb.OUT_DIR, "wsr_serve_api.o")
    wb._run(["hipcc", *wb.COMMON, "-c", os.path.join(wb.CSRC, "wsr_serve_api.cpp"), "-o", obj])
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
