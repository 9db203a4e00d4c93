"""Names of the serving operators in paper_2608_12114_amd.wsr, with and without their library."""
import subprocess
import sys

import paper_2608_12114_amd as package
from paper_2608_12114_amd import wsr, wsr_serve

PUBLIC = [n for n in vars(wsr_serve) if n.startswith(("wsr_", "make_", "serve_")) or n in ("WSR_QKV_NORM", "WSR_QKV_PAIRS")]


def test_every_name_is_reached():
    assert sorted(PUBLIC) == sorted(wsr._SERVE_NAMES) and not wsr._SERVE_NAMES & wsr._STEP_NAMES
    for n in PUBLIC:
        assert getattr(wsr, n) is getattr(wsr_serve, n) is getattr(package, n)


def test_without_the_library():
    """Where libwsr_serve.so is not built, its names are missing attributes whose message says how to build it, and all
    else works as before."""
    script = f"""
import os, sys
sys.path.insert(0, {str(package.__path__[0] + "/..")!r})
exists = os.path.exists
os.path.exists = lambda p: not str(p).endswith("libwsr_serve.so") and exists(p)
from paper_2608_12114_amd import wsr
assert not hasattr(wsr, "no_such_name") and not hasattr(wsr, "wsr_append_qkv") and hasattr(wsr, "wsr_block_norm")
try:
    wsr.wsr_paged_attention
except AttributeError as e:
    assert "is not built" in str(e), e
else:
    raise SystemExit("no error")
"""
    subprocess.run([sys.executable, "-c", script], check=True)
