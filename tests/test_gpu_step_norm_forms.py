"""wsr_block_norm on both sides of each choice of its launch: threads and pieces by the row's width, and residual streams
of 32 MiB or more, which are stored past the caches."""
import pytest
import torch

import step_util as su
from gpu_util import needs_gpu
from test_gpu_step_norm import _call, _check, _inputs

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [504, 520, 2040, 2056, 4088, 4104, 6160, 8184, 8192, 8200, 16384, 16392])
@pytest.mark.parametrize("T", [1, 3])
def test_widths(T, d, kind, dt):
    """One, four, eight and sixteen waves; one, two and four pieces per thread, the last ones partly empty."""
    y, h, vec, gt = _inputs(T, d, dt, kind, True, "token", seed=T + d)
    h_out, x = _call(y, h, T, d, dt, kind, True, gt, 0.9, vec)
    _check(h_out, x, y, h, kind, True, gt, 0.9, vec, dt)


@pytest.mark.parametrize("kind,dt", [("rms", torch.float16), ("layer", torch.bfloat16)])
@pytest.mark.parametrize("T,d", [(511, 8184), (513, 4104), (1100, 8184), (2049, 4096), (16400, 512), (16399, 520), (700, 16376), (520, 16392),
                                 (257, 32768)])
def test_many_tokens(T, d, kind, dt):
    """The first two below 32 MiB of residual stream, the others above."""
    assert (T * d * 4 >= 32 << 20) == (T not in (511, 513))
    y, h, vec, gt = _inputs(T, d, dt, kind, True, "channel", seed=d)
    h_out, x = _call(y, h, T, d, dt, kind, True, gt, 1.1, vec)
    _check(h_out, x, y, h, kind, True, gt, 1.1, vec, dt)


@pytest.mark.parametrize("T,d", [(2051, 4096), (1030, 8192)])
def test_long_streams_in_place(T, d):
    """h_out in place of h, no post norm, strided rows; stored past the caches, read by the next call."""
    dt = torch.bfloat16
    y, h, vec, _ = _inputs(T, d, dt, "rms", False, "none", seed=7)
    stream = torch.zeros((T, d + 16), device="cuda")
    stream[:, :d] = h
    for _ in range(2):
        _, x = _call(y, stream[:, :d], T, d, dt, "rms", False, None, 0.5, vec, h_out=stream[:, :d])
    want, _ = su.block64(y, h, kind="rms", post=False, res=0.5)
    _check(stream[:, :d], x, y, want.float(), "rms", False, None, 0.5, vec, dt)
    assert (stream[:, d:] == 0).all()
