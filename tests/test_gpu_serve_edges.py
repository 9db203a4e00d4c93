"""What the serving operators give at the ends of fp32: infinite scores, squares that overflow, two tokens in one slot."""
import pytest
import torch

from gpu_util import needs_gpu
from test_gpu_serve_append import Case as Append
from test_gpu_serve_paged import BF16, F16, INF, Case

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,G,N,room", [(1, 4, 2, 0), (1, 4, 2, 2000), (5, 4, 2, 0), (7, 8, 1, 2000), (40, 8, 2, 0), (150, 8, 8, 0)])
def test_infinite_scores(D, n, G, N, room):
    """Scores of -inf count for nothing, where all of a row are, the row is as one that sees no key; +inf makes it NaN."""
    c = Case([n, n, n], [n + 90, n + 700, n + 3], N * G, N, D, BF16, page=8, room=room)
    c.q[..., 0] = -c.q[..., 0].abs().clamp(min=0.5)
    c.q[-1, -1, 0] = 1.0                                         # the last row alone meets the keys' infinity with the other sign
    places = torch.arange(c.lens[1], device="cuda")
    at = c.table[1][places // 8].long(), places % 8
    c.k[(*at, 0, 0)] = torch.where(places % 3 != 0, INF, c.k[(*at, 0, 0)].float()).to(BF16)
    last = torch.arange(c.lens[2], device="cuda")
    c.k[c.table[2][last // 8].long(), last % 8, :, 0] = INF
    c.run()
    none = slice(2 * n, 3 * n)
    assert torch.isnan(c.out[-1, -1]).all() and torch.isnan(c.lse[-1, -1])
    c.out[-1, -1], c.lse[-1, -1] = 0.0, -INF
    assert (c.out[none] == 0).all() and torch.isneginf(c.lse[none]).all()
    # the others as if the keys of infinite scores were not there; bounds as in serve_util.paged64
    k, v, q = c.k[at].double(), c.v[at].double(), c.q[n:2 * n, :G].double()
    s = (q @ k[:, 0].nan_to_num(posinf=0.0).t().contiguous()) * c.scale
    see = (places % 3 == 0) & (places < (c.lens[1] - n + 1 + torch.arange(n, device="cuda"))[:, None])
    s = s.masked_fill(~see[:, None], -INF)
    want, lse = torch.softmax(s, -1) @ v[:, 0], torch.logsumexp(s, -1)
    d = (q.abs() @ k[:, 0].abs().nan_to_num(posinf=0.0).t().contiguous()).amax(-1) * c.scale * (D / 8 + 8) * 2.0 ** -24
    r = (len(places) / 16 + 32) * 2.0 ** -24
    bound = (2.0 ** -8 + 2 * d + r)[..., None] * (torch.softmax(s, -1) @ v[:, 0].abs()) + 2.0 ** -8 * want.abs()
    assert ((c.out[n:2 * n, :G].double() - want).abs() <= bound).all()
    assert ((c.lse[n:2 * n, :G].double() - lse).abs() <= d + r + 2.0 ** -22 * (1 + lse.abs())).all()


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_squares_past_the_range(kind):
    """Heads whose squares fp32 does not hold are 0, beside heads that are not."""
    c = Append([2], [9], 4, 2, 64, F16, kind=kind)
    c.q[0, :64] *= 1e25
    c.run()
    assert (c.out[0, 0] == 0).all()
    c.out[0, 0] = c.before[0][0, 0]
    full = c.want()
    full[0][2][0, 0] = False
    c.want = lambda: full
    c.check()


def test_two_tokens_in_one_slot():
    """Every value there is one of theirs, and nothing else is touched."""
    c = Append([1, 1], [5, 5], 4, 2, 64, BF16, page=8)
    c.table[1] = c.table[0]
    c.run()
    page = int(c.table[0, 0])
    alone = []
    for b in range(2):
        o = Append([1, 1], [5, 5], 4, 2, 64, BF16, page=8)
        o.table[:] = -1
        o.table[b] = c.table[0]
        o.run()
        alone.append((o.kc, o.vc))
    for got, a, b, old in zip((c.kc, c.vc), alone[0], alone[1], c.before[1:]):
        assert ((got[page, 4] == a[page, 4]) | (got[page, 4] == b[page, 4])).all()
        got[page, 4] = old[page, 4]
        assert torch.equal(got.view(torch.int16), old.view(torch.int16))
