"""wsr_token_logprobs against its definition in 64 bits: both forms, ties, masked and broken logits, temperatures, rows
that are odd in length and place."""
import math

import pytest
import torch

import serve_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
INF, NAN = math.inf, math.nan


class Case:
    def __init__(self, logits, tokens, n_top, temps=None, stride=None):
        R, V = logits.shape
        self.logits, self.tokens, self.n_top, self.temps = logits, tokens, n_top, temps
        new = lambda *s, to=torch.float32: torch.full(s, 99, dtype=to, device="cuda")  # noqa: E731
        self.logp, self.rank, self.entropy = new(R), new(R, to=torch.int32), new(R)
        self.top, self.top_logp = new(R, n_top, to=torch.int32), new(R, n_top)
        self.dev_tokens = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        self.dev_temps = None if temps is None else torch.tensor(temps, device="cuda")
        self.fields = dict(n_rows=R, vocab=V, n_top=n_top, logits=logits, row_stride=4 * logits.stride(0), tokens=self.dev_tokens,
                           temperature=self.dev_temps, logp=self.logp, rank=self.rank, entropy=self.entropy, top=self.top,
                           top_logp=self.top_logp)

    def run(self, sync=True, on=None, **over):
        self.p = wsr.make_logprobs(**{**self.fields, **over})
        self.ws = torch.full((wsr.wsr_logprobs_workspace_bytes(self.p),), 255, dtype=torch.uint8, device="cuda")
        wsr.wsr_token_logprobs(self.p, self.ws, self.ws.numel(), on or stream())
        if sync:
            torch.cuda.synchronize()

    def check(self, rows=None):
        V = self.logits.shape[1]
        # values past fp32's range round to infinities: lowest / 0.3 is -1.13e39
        near = lambda got, want: got == float(torch.tensor(want).to(torch.float32)) or abs(got - want) <= su.logp_bound(V, want)  # noqa: E731
        for r in rows if rows is not None else range(self.logits.shape[0]):
            T = 1.0 if self.temps is None else self.temps[r]
            logp, rank, entropy, top, top_logp = su.logprobs64(self.logits[r], self.tokens[r], T, self.n_top)
            assert self.rank[r] == rank and self.top[r].tolist() == top, (r, self.rank[r], rank, self.top[r].tolist(), top)
            assert near(float(self.logp[r]), logp), (r, float(self.logp[r]), logp)
            assert all(map(near, self.top_logp[r].tolist(), top_logp)), (r, self.top_logp[r].tolist(), top_logp)
            assert abs(float(self.entropy[r]) - entropy) <= su.entropy_bound(V, entropy), (r, float(self.entropy[r]), entropy)


def _normal(R, V, seed=0, std=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(R, V, generator=g, device="cuda") * std


@pytest.mark.parametrize("n_top", [0, 1, 2, 20, 63, 64])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 4095, 4096, 4097, 50257])
def test_matches_definition(V, n_top):
    R = 5
    c = Case(_normal(R, V, V + n_top), [(r * 7919) % V for r in range(R)], n_top, [1.0, 0.5, 1.7, 0.0, 3.0])
    c.run()
    c.check()


@pytest.mark.parametrize("R,V,n_top", [(1, 128256, 5), (3, 151937, 64), (700, 5003, 11), (2100, 4100, 3), (2100, 9001, 0), (40, 128256, 1)])
def test_few_and_many_rows(R, V, n_top):
    c = Case(_normal(R, V, R), [(r * 104729) % V for r in range(R)], n_top)
    c.run()
    c.check([0, 1, R // 2, R - 2, R - 1] if R > 5 else None)


@pytest.mark.parametrize("V", [64, 777, 20000])
@pytest.mark.parametrize("n_top", [1, 7, 64])
def test_ties_go_to_the_lowest_index(V, n_top):
    rows = [torch.zeros(V), torch.arange(V).remainder(3).float(), -torch.arange(V).remainder(5).float(),
            torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0), torch.full((V,), -1e30), torch.arange(V).float() / V,
            -torch.arange(V).float() / V]
    c = Case(torch.stack(rows).cuda(), [V // 2, V - 1, 0, 1, V - 1, V // 3, V // 3], n_top)
    c.run()
    c.check()


@pytest.mark.parametrize("V", [5, 300, 9000])
def test_masked_and_broken_logits(V):
    """Rows held to a few tokens, NaN and infinities of both signs, rows with nothing to draw, tokens outside the vocabulary."""
    x = _normal(12, V, 5)
    keep = torch.zeros(V, dtype=torch.bool, device="cuda")
    keep[[1, V // 2, V - 1]] = True
    x[0, ~keep] = -INF
    x[1] = -INF
    x[2] = NAN
    x[3, ::2] = NAN
    x[4, V // 2] = INF
    x[5, [0, V - 1]] = INF
    x[6, :] = torch.finfo(torch.float32).min
    x[7, ~keep] = torch.finfo(torch.float32).min
    x[8, 1:] = -INF
    x[9, 3] = NAN
    x[10, 2] = torch.finfo(torch.float32).max
    c = Case(x, [V // 2, 3, 2, 2, V // 2, 1, V - 1, 0, 2, 3, V, -1], min(V, 9) + 1, [1.0, 0.7, 1.0, 2.0, 0.0, 1.0, 1.0, 0.3, 1.0, 1.0, 1.0, 1.0])
    c.run()
    c.check()


def test_temperatures():
    """Zero and what is not above it, large and infinite ones."""
    temps = [0.0, -1.0, NAN, 1e-3, 100.0, 1e30, INF, 1e-30]
    c = Case(_normal(8, 3000, 3), [int(v) for v in _normal(8, 3000, 3).argmax(-1).tolist()], 6, temps)
    c.temps = [0.0 if not t > 0 else t for t in temps]
    c.run()
    c.check()


def test_temperatures_near_zero():
    """Those whose inverse fp32 does not hold count as the smallest normal one: the largest logits share the probability."""
    x = _normal(5, 3000, 7)
    x[:, 11] = x[:, 2999] = x.max() + 1
    c = Case(x, [11, 2999, 0, 2999, 11], 3, [2.0 ** -149, 1e-40, 1e-39, 2.0 ** -126, 1.5e-38])
    c.run()
    c.check()
    assert (c.logp[[0, 1, 3, 4]] + 0.6931471805599453).abs().max() < 1e-6 and (c.entropy - 0.6931471805599453).abs().max() < 1e-6


def test_rows_anywhere():
    """Rows that start at any 4 bytes and are apart; NaN between them is not read."""
    wide = torch.full((9, 5009), NAN, device="cuda")
    x = wide.flatten()[3:3 + 8 * 5009].view(8, 5009)[:, :5001]
    x.copy_(_normal(8, 5001))
    c = Case(x, list(range(8)), 10)
    c.run()
    c.check()


def test_same_row_for_all_and_left_out_outputs():
    x = _normal(1, 7000).expand(6, 7000)
    c = Case(x, [0, 1, 2, 3, 4, 6999], 4)
    c.run(row_stride=0)
    c.check()
    c.logp.fill_(5.0), c.rank.fill_(5)
    want = c.top.clone()
    c.top.fill_(-7)
    c.run(row_stride=0, tokens=None, logp=None, rank=None, entropy=None, top_logp=None)
    assert torch.equal(c.top, want) and (c.logp == 5.0).all() and (c.rank == 5).all()
    c.run(row_stride=0, n_top=0, top=None, top_logp=None, entropy=None)
    c.run(row_stride=0)
    c.check()


@pytest.mark.parametrize("spread", [1e-3, 40.0])
def test_flat_and_peaked_rows(spread):
    c = Case(_normal(4, 32000, 9, spread), [5, 6, 7, 8], 20)
    c.run()
    c.check()
