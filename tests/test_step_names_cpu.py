"""Names of the step operators in paper_2608_12114_amd.wsr, with and without their library."""
import subprocess
import sys

import pytest

import paper_2608_12114_amd as package
from paper_2608_12114_amd import wsr, wsr_step

PUBLIC = [n for n in vars(wsr_step) if n.startswith(("wsr_", "make_", "step_")) or n in ("WSR_NORM_RMS", "WSR_NORM_LAYER", "WSR_BLOCK_POST")]


def test_every_name_is_reached():
    assert sorted(PUBLIC) == sorted(wsr._STEP_NAMES)
    for n in PUBLIC:
        assert getattr(wsr, n) is getattr(wsr_step, n)


def test_other_names_are_no_attributes():
    for n in ("no_such_name", "_no_such_name", "LIB_PATH_", "annotations_"):
        assert not hasattr(wsr, n)
        with pytest.raises(AttributeError, match=n):
            getattr(wsr, n)


def test_without_the_library():
    """Where libwsr_step.so is not built, its names are missing attributes whose message says how to build it, and all
    else works as before."""
    script = f"""
import os, sys
sys.path.insert(0, {str(package.__path__[0] + "/..")!r})
exists = os.path.exists
os.path.exists = lambda p: not str(p).endswith("libwsr_step.so") and exists(p)
from paper_2608_12114_amd import wsr
assert not hasattr(wsr, "no_such_name") and not hasattr(wsr, "wsr_block_norm") and hasattr(wsr, "wsr_decode_sweep_mma")
assert getattr(wsr, "anything", 3) == 3
try:
    wsr.wsr_block_norm
except AttributeError as e:
    assert "is not built" in str(e), e
else:
    raise SystemExit("no error")
"""
    subprocess.run([sys.executable, "-c", script], check=True)
