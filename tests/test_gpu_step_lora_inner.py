"""The inner vectors A x of wsr_lora_sweep in 16-bit terms: entries of one token that differ widely in size, and infinities
beside finite entries past the type's range."""
import math

import pytest
import torch

import step_util as su
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


def _within(c):
    """Every output within the roundings of its own terms: fp32 sums, inner vectors of 22 bits."""
    for m in c.mods:
        y, mag = su.lora64(m["x"], m["a"], m["b"], c.ids.tolist(), None, None if c.scales is None else c.scales.tolist(), m["src"])
        bound = (su.U32 * (8 + 2 * math.sqrt(m["K"]) + 2 * math.sqrt(c.rank)) + 2.0 ** -22) * mag
        assert (mag > 0).all()
        err = (m["y"].double() - y).abs()
        assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("up,down", [(4, -8), (8, -12), (13, -13), (14, -14)])
@pytest.mark.parametrize("T,n,rank", [(1, 1, 16), (5, 2, 16), (20, 3, 12), (20, 2, 80), (130, 5, 24)])
def test_ranks_of_different_size(T, n, rank, up, down, dt):
    """Half of the ranks are 2^(up - down) larger than the others, and every other row of B reads the small ones alone: their
    share of y keeps its bits."""
    c = Case([(96, 64), (70, 200)], T, n, rank, dt, seed=rank + up, y0="none")
    for m in c.mods:
        m["a"][:, ::2] *= 2.0 ** up
        m["a"][:, 1::2] *= 2.0 ** down
        m["b"][:, ::2, ::2] = 0.0
    c.run()
    _within(c)


@pytest.mark.parametrize("dt,a,x", [(torch.float16, -9, -9), (torch.float16, -13, -13), (torch.float16, 12, 12), (torch.float16, -12, 10),
                                    (torch.bfloat16, -40, -40), (torch.bfloat16, 50, 40)])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_small_and_large_inner_vectors(T, a, x, dt):
    c = Case([(96, 64), (33, 520)], T, 2, 16, dt, seed=12, y0="none")
    for m in c.mods:
        m["a"].mul_(2.0 ** a), m["x"].mul_(2.0 ** x)
    c.run()
    _within(c)
