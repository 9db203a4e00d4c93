"""Scales that paged attention takes: the kernels' powers of two need scale times log2 e, which fp32 holds up to 2^127."""
import math

import pytest

from paper_2608_12114_amd import wsr
from test_serve_abi_cpu import A, ARG, SIZE, L, _paged


@pytest.mark.parametrize("scale,st", [(2.0 ** 127, SIZE), (2.5e38, ARG), (3.4e38, ARG), (math.inf, ARG), (1e-45, SIZE), (0.0, ARG), (-1.0, ARG)])
def test_scales(scale, st):
    """SIZE: taken, as far as the workspace, which has no bytes here."""
    assert L.wsr_paged_attention(_paged(scale=scale), A, 0, None) == st
    assert (wsr.wsr_paged_workspace_bytes(_paged(scale=scale)) > 0) == (st == SIZE)
