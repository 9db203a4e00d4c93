"""The inner vectors A x of wsr_lora_sweep in 16-bit terms: entries of one token that differ widely in size, and infinities
beside finite entries past the type's range."""
import pytest
import torch

from gpu_util import needs_gpu
from test_gpu_step_lora import Case

pytestmark = [pytest.mark.gpu, needs_gpu]
INF = float("inf")


@pytest.mark.parametrize("T", [1, 9, 33, 100])
@pytest.mark.parametrize("rank", [16, 80])
def test_an_infinite_entry_beside_large_ones(T, rank):
    """v = (inf, 2^17, 0 ...), the second past the end of f16: the infinity decides, whatever the sign of the second's weight."""
    c = Case([(64, 512), (40, 1 << 17)], T, 1, rank, torch.float16, seed=50, y0="none", scales=False)
    for m in c.mods:
        for name in ("x", "a", "b"):
            m[name].zero_()
        m["x"][:, 0], m["x"][:, 1] = 1.0, 2.0 ** 15
        m["a"][0, 0, 0], m["a"][0, 1, 1] = INF, 4.0
        m["b"][0, :, 0], m["b"][0, :, 1] = 1.0, 1.0
        m["b"][0, 1::2, 0], m["b"][0, ::3, 1] = -1.0, -1.0
    c.run()
    for m in c.mods:
        assert (m["y"][:, ::2] == INF).all() and (m["y"][:, 1::2] == -INF).all()
