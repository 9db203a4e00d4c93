"""Properties of the serving operators' compiled gfx950 code, checked on the CPU from the device assembly that the build's
own flags produce: no packed fp32 arithmetic and no scratch memory in any kernel."""
import os
import re
import subprocess

import pytest

from paper_2608_12114_amd import build as wb
from paper_2608_12114_amd import build_serve as wbs


@pytest.fixture(scope="module", params=wbs.KERNEL_FILES)
def asm(request, tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "k.s"
    subprocess.run(["hipcc", *wb.COMMON, *wb.DEVICE, "-S", "--cuda-device-only", os.path.join(wb.CSRC, request.param), "-o",
                    str(out)], check=True, capture_output=True)
    return out.read_text()


def test_no_packed_fp32(asm):
    assert not re.findall(r"\bv_pk_(fma|add|mul|mov)_f32\b", asm)


def test_no_scratch(asm):
    sizes = [int(v) for v in re.findall(r"\.private_segment_fixed_size:\s+(\d+)", asm)]
    assert sizes and all(v == 0 for v in sizes)
