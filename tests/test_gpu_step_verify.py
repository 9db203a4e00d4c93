"""wsr_verify_drafts against its rules in 64 bits.  Decisions nearer than 1e-5 (relative) to a tie may fall
either way in 32 bits; the tests count them and compare every other sequence exactly."""
import math

import pytest
import torch

import step_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
INF, NAN = float("inf"), float("nan")


class Case:
    def __init__(self, B, n, V, seed=0, points=False, temps=(1.0, 0.7, 0.0, 1.3), counts=None, spread=2.0, near=0.6, pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.B, self.n, self.V = B, n, V
        self.target = (r(B, n + 1, V + pad) * spread)[..., :V]
        self.draft = None
        drafted = self.target[:, :n] + near * r(B, n, V)
        if not points:
            self.draft = torch.empty((B, n, V + pad), device="cuda")[..., :V]
            self.draft.copy_(drafted)
        self.temps = None if temps is None else torch.tensor([temps[b % len(temps)] for b in range(B)], device="cuda")
        heat = torch.ones(B, device="cuda") if temps is None else self.temps
        race = heat[:, None, None] * torch.empty((B, n, V), device="cuda").exponential_(generator=g).log_()
        self.tokens = (drafted - race).argmax(-1).to(torch.int32) if n else torch.zeros((B, 0), dtype=torch.int32, device="cuda")
        self.counts = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        self.uniform = torch.rand((B, n), generator=g, device="cuda")
        self.noise = torch.empty((B, V + pad), device="cuda").exponential_(generator=g).clamp_(min=1e-30)[:, :V]

    def run(self, logp=True, sync=True):
        B, n = self.B, self.n
        if not hasattr(self, "out"):
            self.out = torch.full((B, n + 1), -7, dtype=torch.int32, device="cuda")
            self.accepted = torch.full((B,), -7, dtype=torch.int32, device="cuda")
            self.logp = torch.full((B, n + 1), NAN, device="cuda")
        st = lambda t, d: 0 if t is None else 4 * t.stride(d)  # noqa: E731
        v = wsr.make_verify(
            n_seqs=B, n_drafts=n, vocab=self.V, target=self.target, target_seq_stride=st(self.target, 0),
            target_row_stride=st(self.target, 1), draft=self.draft, draft_seq_stride=st(self.draft, 0),
            draft_row_stride=st(self.draft, 1), tokens=self.tokens, counts=self.counts, temperature=self.temps,
            uniform=self.uniform, noise=self.noise, noise_seq_stride=st(self.noise, 0), out=self.out, accepted=self.accepted,
            logp=self.logp if logp else None)
        if not hasattr(self, "ws"):
            self.ws = torch.full((wsr.wsr_verify_workspace_bytes(v),), 255, dtype=torch.uint8, device="cuda")
        wsr.wsr_verify_drafts(v, self.ws, self.ws.numel(), stream())
        if sync:
            torch.cuda.synchronize()

    def check(self, skip=0.05):
        counts = [self.n] * self.B if self.counts is None else self.counts.tolist()
        temps = [1.0] * self.B if self.temps is None else self.temps.tolist()
        want = su.verify64(self.target, self.draft, self.tokens.tolist(), counts, temps, self.uniform.tolist(), self.noise)
        out, acc, logp = self.out.tolist(), self.accepted.tolist(), self.logp.tolist()
        skipped = 0
        for b, (o, a, lp, near) in enumerate(want):
            if near < 1e-5:
                skipped += 1
                continue
            assert (out[b], acc[b]) == (o, a), (b, out[b], o, near)
            for x, y in zip(logp[b], lp):
                assert x == y or abs(x - y) <= 2e-6 * abs(y) + 4e-6, (b, x, y)
        assert skipped <= skip * self.B + 1


@pytest.mark.parametrize("points", [False, True])
@pytest.mark.parametrize("B,n,V", [(1, 0, 1), (3, 1, 2), (1, 4, 1000), (9, 3, 8191), (5, 2, 8193), (4, 7, 32003), (2, 5, 128256),
                                   (33, 4, 517), (2, 63, 100)])
def test_matches_rules(B, n, V, points):
    c = Case(B, n, V, seed=B + V, points=points)
    c.run()
    c.check()


def test_counts_strides_and_no_temperatures():
    c = Case(8, 4, 3001, seed=1, temps=None, counts=[0, 1, 2, 3, 4, -1, 9, 2], pad=5)
    c.target[0, 1:], c.draft[0] = NAN, NAN                  # rows beyond the counts are not looked at
    c.run()
    c.check()


def test_equal_models_accept_everything():
    c = Case(16, 5, 700, seed=2, near=0.0, temps=(1.0, 0.5))
    c.run()
    assert (c.accepted == 5).all()
    c.check()


def test_a_draft_the_target_cannot_draw_is_refused():
    c = Case(6, 3, 400, seed=3, temps=(1.0, 0.0))
    for b in range(6):
        c.target[b, 1, int(c.tokens[b, 1])] = -INF
    c.uniform.zero_()
    c.run()
    assert (c.accepted <= 1).all()
    c.check()


def test_drafts_outside_the_vocabulary_are_refused():
    c = Case(4, 3, 100, seed=4)
    c.tokens[:, 1] = torch.tensor([-1, 100, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64, device="cuda").to(torch.int32)
    c.run()
    assert (c.accepted <= 1).all()
    c.check(skip=0.5)


def test_greedy_ties_take_the_lowest_index():
    V = 20000
    c = Case(3, 2, V, seed=5, temps=(0.0,))
    c.target[:] = -1.0
    c.draft[:] = -1.0
    for b, i in enumerate((0, 8190, 13333)):
        c.target[b, :, i] = 2.0
        c.target[b, :, i + 1:i + 4000:7] = 2.0
        c.draft[b, :, i] = 1.0
        c.tokens[b, 0], c.tokens[b, 1] = i, i + 1
    c.run()
    assert c.accepted.tolist() == [1, 1, 1]
    assert c.out.tolist() == [[i, i, -1] for i in (0, 8190, 13333)]
    assert (c.logp == 0).all()


def test_equal_race_scores_take_the_lowest_index():
    V = 17000
    c = Case(2, 0, V, seed=6, temps=(1.0,))
    c.target[:] = 0.0
    c.noise[:] = 1.0
    c.noise[0, 9000:9100] = 0.5
    c.run()
    assert c.out.tolist() == [[9000], [0]]


def test_masked_infinite_and_empty_rows():
    V = 9000
    c = Case(6, 1, V, seed=7, temps=(1.0,))
    c.target[0, :, ::2] = NAN                               # NaN counts as -inf
    c.target[1, 0] = -INF                                   # nothing to draw: token -1
    c.target[2, 0], c.target[2, 0, 77] = -INF, -3.0         # one token left
    c.target[3, 0, 5], c.target[3, 0, 8999] = INF, INF      # they share everything
    c.target[4, 0] = torch.finfo(torch.float32).min         # all at the type's lowest value: uniform
    c.draft[5, 0] = -INF                                    # a draft that had no distribution
    c.run()
    c.check(skip=0.5)
    assert c.out[1].tolist() == [-1, -1] and c.accepted[1] == 0 and c.logp[1, 0] == -INF


def test_same_distribution_refused_falls_back_to_the_target():
    """uniform = 1 (out of its range) refuses a draft although p = q: the race is over p then."""
    c = Case(2, 1, 300, seed=8, near=0.0, temps=(1.0,))
    c.uniform.fill_(1.0)
    c.run()
    assert (c.accepted == 0).all() and ((c.out[:, 0] >= 0) & (c.out[:, 0] < 300)).all()
    c.check(skip=1.0)


def test_race_draws_in_proportion():
    """20000 one-token vocabularies' draws: each token's share within five standard deviations."""
    B, V = 20000, 6
    c = Case(B, 0, V, seed=9, temps=(1.0,))
    c.target[:] = torch.log(torch.tensor([0.3, 0.05, 0.2, 0.25, 0.15, 0.05], device="cuda"))
    c.run()
    share = torch.bincount(c.out[:, 0].long(), minlength=V).double() / B
    for p, s in zip([0.3, 0.05, 0.2, 0.25, 0.15, 0.05], share.tolist()):
        assert abs(p - s) <= 5 * math.sqrt(p * (1 - p) / B)


def test_without_logp_other_stream_and_graph():
    c = Case(7, 3, 40000, seed=10)
    c.run()
    want = c.out.clone(), c.accepted.clone(), c.logp.clone()
    c.logp.fill_(5.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.run(logp=False)
    assert torch.equal(c.out, want[0]) and torch.equal(c.accepted, want[1]) and (c.logp == 5).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run(sync=False)
    for k in range(4):
        c.uniform.copy_(torch.rand(7, 3, device="cuda"))
        c.out.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        c.check(skip=0.2)
        got = c.out.clone()
        c.run()
        assert torch.equal(got, c.out)


def test_infinite_temperature_is_even():
    """All that can be drawn is equally likely; with an infinite logit, that one alone."""
    c = Case(4, 2, 300, seed=31, temps=(INF, INF))
    c.target[:, :, 5] = -INF
    c.target[1, 0, 9] = INF
    c.run()
    token, logp = c.out[:, 0].tolist(), c.logp[:, 0].tolist()
    assert 5 not in c.out.flatten().tolist()
    for b in (0, 2, 3):
        assert abs(logp[b] + 5.7004435733906869) < 1e-5, logp       # log 299
    assert token[1] == 9 and logp[1] == 0
