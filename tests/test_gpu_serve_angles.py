"""wsr_append_qkv's angles against exact arithmetic: position times frequency as whole numbers, a turn of 60 digits."""
import functools
import math
from fractions import Fraction

import pytest
import torch

from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
PI = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164, 10 ** 70)
BITS = 200
TURNS = int(2 ** BITS / (2 * PI))             # 2^200 / (2 pi)


def turned(position, frequency):
    """Sine and cosine of position * frequency, from its part of a turn, which has more than 100 bits."""
    m, e = math.frexp(frequency)
    part = (position * int(m * 2 ** 24) * TURNS >> 24 - e) % 2 ** BITS
    part = part - 2 ** BITS if part >= 2 ** (BITS - 1) else part
    quarter = round(Fraction(part, 2 ** (BITS - 2)))           # the nearest quarter turn, and what is left
    rest = float(Fraction(part - quarter * 2 ** (BITS - 2), 2 ** BITS) * 2 * PI)
    s, c = math.sin(rest), math.cos(rest)
    return ((s, c), (c, -s), (-s, -c), (-c, s))[quarter % 4]


FREQS = [float(torch.tensor(f)) for f in (1.0, 2 ** -0.5, 0.4, 0.9, 0.61, 0.8317, 0.55, 0.3)]


@functools.lru_cache
def near_quarters(far):
    """Positions up to `far` at which one of the angles is within 2^-14 of whole quarter turns."""
    return [p for p in range(max(0, far - (1 << 15)), far + 1) if any(min(map(abs, turned(p, f))) < 2 ** -14 for f in FREQS)]


def test_definition():
    for p, f in ((1, 1.0), (-3, 0.5), (100, 0.25), (7, 2.0)):
        assert turned(p, f) == pytest.approx((math.sin(p * f), math.cos(p * f)), abs=1e-14)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("far", [1000, 1 << 24, (1 << 31) - 1])
def test_angles_near_whole_quarters(far, pairs):
    """A sine (cosine) near 0 shows what an angle has lost: in bf16 it is off by 2^-8 of itself for its rounding and by 8 half
    steps of fp32 for the rest's, the constant's and the series', all relative to it, whatever the position."""
    freqs, (D, rot) = FREQS, (64, 16)
    found = near_quarters(far) + [far, -far]
    T = len(found)
    if far > 1000:
        assert T > 10
    x = torch.zeros(T, D, device="cuda")
    x[:, slice(1, rot, 2) if pairs else slice(rot // 2, rot)] = 1.0       # pairs (0, 1) become (-sin, cos)
    out = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor(found, dtype=torch.int32, device="cuda")
    lens, f32 = torch.ones(T, dtype=torch.int32, device="cuda"), torch.tensor(freqs, device="cuda")
    wsr.wsr_append_qkv(wsr.make_qkv(fmt=wsr.WSR_BF16, flags=wsr.WSR_QKV_PAIRS if pairs else 0, n_heads=1, head_dim=D, rot_dim=rot,
                                    n_seqs=T, n_tokens=T, q=x, q_tok_stride=4 * D, freqs=f32, positions=at, pos_axis_stride=4 * T,
                                    lens=lens, q_out=out, q_out_tok_stride=2 * D, q_out_head_stride=2 * D), stream())
    torch.cuda.synchronize()
    got = out[:, :rot].double().cpu()
    got = got.view(T, rot // 2, 2) if pairs else got.view(T, 2, rot // 2).transpose(1, 2)
    want = torch.tensor([[turned(p, f) for f in freqs] for p in found], dtype=torch.float64) * torch.tensor([-1.0, 1.0])
    assert ((got - want).abs() <= (2.0 ** -8 + 8 * 2.0 ** -24) * want.abs() + 2.0 ** -50).all()
