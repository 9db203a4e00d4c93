"""Projections without rows, and of no terms, beside others in one adapters' sweep: with null pointers throughout, in the
form of one launch and in that of two."""
import pytest
import torch

from gpu_util import needs_gpu
from paper_2608_12114_amd import wsr
from test_gpu_step_lora import FMT, Case

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,n,rank", [(2, 2, 8), (5, 3, 24), (30, 4, 16), (140, 6, 8)])
def test_null_pointers(T, n, rank, dt):
    c = Case([(72, 512), (0, 4096), (33, 0), (0, 8), (200, 136)], T, n, rank, dt, seed=T)
    for i in (1, 3):
        c.table[i] = wsr.make_loras([dict(fmt=FMT[dt], rank=64, M=0, K=1 << 20)])[0]
    c.table[2].a, c.table[2].x = None, None                 # K = 0: nothing to read
    c.run()
    c.check()
