"""NaN among the scores of wsr_prefix_attention: out and lse of the rows that have them are NaN, the others' are as they
would be without; in the split form of one, two and four waves over rows and in the whole form."""
import math

import pytest
import torch

import step_util as su
from gpu_util import needs_gpu
from test_gpu_step_attn import NAN, Case

pytestmark = [pytest.mark.gpu, needs_gpu]
FORMS = [([1, 2, 1], [5, 300, 64], 700, 8, 2), ([3] * 4, [9] * 4, 70, 16, 4), ([5, 30], [40, 700], 0, 8, 2),
         ([130, 1, 64, 300], [130, 90, 64, 301], 193, 128, 64)]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("counts,lens,P,H,N", FORMS)
def test_a_nan_in_a_query(counts, lens, P, H, N, D, dt):
    c = Case(counts, lens, P, H, N, D, dt, seed=40)
    rows = torch.zeros(c.q.shape[:2], dtype=torch.bool, device="cuda")
    rows[0, 1], rows[c.starts[1], H - 1], rows[-1, 0] = True, True, True
    good = c.q.clone()
    c.q[rows, 5] = NAN
    c.run()
    assert torch.isnan(c.out[rows]).all() and torch.isnan(c.lse[rows]).all()
    out, lse, mag = su.attn64(good, c.kp, c.vp, c.k, c.v, c.starts, c.lens, c.scale)
    u = su.U16[dt]
    bound = (u + 1e-4) * mag + u * out.abs() + 64 * 2.0 ** -25 * (1 + mag.amax(-1, keepdim=True))
    assert ((c.out.double() - out).abs() <= bound)[~rows].all()
    assert ((c.lse.double() - lse).abs() <= 2e-5)[~rows].all()


@pytest.mark.parametrize("counts,lens,H,N", [([2, 1], [4, 6], 8, 2), ([300, 300], [300, 300], 64, 64)])
def test_all_keys_nan(counts, lens, H, N):
    """A row whose every key is NaN has seen keys: NaN.  One that sees none has not: zeros and -inf."""
    c = Case(counts, [lens[0], 0], 0, H, N, 64, torch.bfloat16, seed=41, S=max(lens))
    c.k[0] = NAN
    c.run()
    n = counts[0]
    assert torch.isnan(c.out[:n]).all() and torch.isnan(c.lse[:n]).all()
    assert (c.out[n:] == 0).all() and (c.lse[n:] == -math.inf).all()
