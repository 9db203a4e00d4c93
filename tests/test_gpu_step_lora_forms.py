"""wsr_lora_sweep in each form of its second launch: units of 64 and of 128 rows for up to 16 tokens, outputs of 32 MiB or
more, which go past the caches; whole and cut last tiles, broken weights, several windows of ranks."""
import math

import pytest
import torch

import step_util as su
from gpu_util import needs_gpu
from test_gpu_step_lora import Case

pytestmark = [pytest.mark.gpu, needs_gpu]
MIB32 = 32 << 20


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [49151, 49152, 49161, 60001])
@pytest.mark.parametrize("T,n,rank,ranks", [(1, 1, 72, None), (5, 3, 16, [16, 8, 3]), (16, 14, 8, None), (9, 2, 80, [80, 65])])
def test_units_of_rows_for_few_tokens(T, n, rank, ranks, rows, dt):
    """Below and from 49152 rows on, spread over three projections that end inside a unit."""
    assert T * rows * 4 < MIB32
    c = Case([(40000, 72), (133, 4104), (rows - 40133, 136)], T, n, rank, dt, seed=T + rank, ranks=ranks)
    if T > 2:
        c.ids[2] = -1
    c.run()
    c.check()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("y0", ["apart", "in place", "none"])
@pytest.mark.parametrize("T,n,rank,rows", [(3, 2, 24, 2800003), (16, 5, 8, 524303), (40, 4, 12, 209731), (64, 64, 4, 131075),
                                           (100, 7, 16, 84001), (333, 3, 70, 25201)])
def test_outputs_past_the_caches(T, n, rank, rows, y0, dt):
    assert T * rows * 4 >= MIB32
    c = Case([(rows - 77, 64), (77, 1032)], T, n, rank, dt, seed=T, y0=y0, ranks=[rank - i % 3 for i in range(n)])
    c.ids[1::5] = -1
    c.run()
    c.check()


@pytest.mark.parametrize("T,n,rank,rows", [(9, 4, 16, 50003), (16, 4, 8, 530003), (40, 5, 8, 210003), (200, 30, 12, 42003)])
@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
def test_broken_adapters_in_wide_projections(T, n, rank, rows, dt):
    c = Case([(rows, 128)], T, n, rank, dt, seed=20)
    c.ids[:n] = torch.arange(n, dtype=torch.int32)
    c.ids[n] = -1
    m = c.mods[0]
    m["b"][1, ::3, 0], m["b"][1, 1::3, rank - 1], m["a"][2, 1, 5] = float("nan"), float("inf"), float("inf")
    c.run()
    whole = (c.ids != 1) & (c.ids != 2)
    y, mag = su.lora64(m["x"], m["a"], m["b"], c.ids.tolist(), None, c.scales.tolist(), m["src"])
    bound = su.U32 * (8 + 2 * math.sqrt(m["K"]) + 2 * math.sqrt(rank)) * mag
    assert ((m["y"].double() - y).abs() <= bound)[whole].all()
    assert torch.isnan(m["y"][c.ids == 1][:, ::3]).all() and torch.isinf(m["y"][c.ids == 1][:, 1::3]).all()
    assert not torch.isfinite(m["y"][c.ids == 2]).any()


@pytest.mark.parametrize("T,rows", [(12, 50001), (12, 800001), (80, 105001)])
def test_steady_bits_of_wide_projections(T, rows):
    c = Case([(rows, 264)], T, 5, 16, torch.bfloat16, seed=13, y0="in place")
    base = c.mods[0]["y"].clone()
    c.run()
    want = c.mods[0]["y"].clone()
    for _ in range(2):
        c.mods[0]["y"].copy_(base)
        c.run()
        assert torch.equal(c.mods[0]["y"], want)
