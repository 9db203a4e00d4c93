"""wsr_prefix_attention against its formula in 64 bits: both forms of the kernel, ragged sequences and drafts, rows
that see nothing, keys past the lengths full of NaN, other layouts, offsets past 4 GiB, a captured graph."""
import pytest
import torch

import step_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
FMT = {torch.float16: wsr.WSR_F16, torch.bfloat16: wsr.WSR_BF16}
NAN = float("nan")


class Case:
    def __init__(self, counts, lens, P, H, N, D, dt, seed=0, S=None, scale=None, head_major=False, prefix=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt)  # noqa: E731
        B, T = len(counts), sum(counts)
        S = max([1] + list(lens)) if S is None else S
        self.counts, self.lens, self.scale = counts, list(lens), D ** -0.5 if scale is None else scale
        self.starts = [sum(counts[:i]) for i in range(B + 1)]
        self.q = (r(T, H, D).float() * 2).to(dt)
        if head_major:          # (heads, tokens, dim) in memory
            kv = lambda *s: r(s[0], s[2], s[1], s[3]).transpose(1, 2)  # noqa: E731
            self.kp, self.vp = r(N, max(P, 1), D).transpose(0, 1)[:P], r(N, max(P, 1), D).transpose(0, 1)[:P]
            self.k, self.v = kv(B, S, N, D), kv(B, S, N, D)
        else:
            self.kp, self.vp, self.k, self.v = r(max(P, 1), N, D)[:P], r(max(P, 1), N, D)[:P], r(B, S, N, D), r(B, S, N, D)
        if prefix is not None:
            self.kp, self.vp = prefix
        for b, n in enumerate(self.lens):                      # what lies past a sequence's keys
            self.k[b, max(n, 0):], self.v[b, max(n, 0):] = NAN, NAN
        self.dev_starts = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.dev_lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.out = torch.full((T, H, D), NAN, dtype=dt, device="cuda")
        self.lse = torch.full((T, H), NAN, device="cuda")
        st = lambda t, d: t.stride(d) * 2  # noqa: E731
        self.attn = wsr.make_attn(
            fmt=FMT[dt], n_heads=H, n_kv_heads=N, head_dim=D, n_seqs=B, n_tokens=T, max_len=S, scale=self.scale, q=self.q,
            q_tok_stride=st(self.q, 0), q_head_stride=st(self.q, 1), k_prefix=self.kp if P else None, v_prefix=self.vp if P else None,
            prefix_len=P, prefix_tok_stride=st(self.kp, 0), prefix_head_stride=st(self.kp, 1), k=self.k, v=self.v,
            kv_seq_stride=st(self.k, 0), kv_tok_stride=st(self.k, 1), kv_head_stride=st(self.k, 2), starts=self.dev_starts,
            lens=self.dev_lens, out=self.out, out_tok_stride=st(self.out, 0), out_head_stride=st(self.out, 1), lse=self.lse)
        self.ws = torch.full((wsr.wsr_attn_workspace_bytes(self.attn),), 255, dtype=torch.uint8, device="cuda")

    def run(self, sync=True):
        wsr.wsr_prefix_attention(self.attn, self.ws, self.ws.numel(), stream())
        if sync:
            torch.cuda.synchronize()

    def check(self):
        out, lse, mag = su.attn64(self.q, self.kp, self.vp, self.k, self.v, self.starts, self.lens, self.scale)
        u = su.U16[self.q.dtype]
        # probabilities rounded to 16 bits (against sum p |v|) and the result once more; scores and sums in
        # fp32 add their share of 2^-24 terms; halves below 2^-14 round in steps of 2^-24
        small = 2.0 ** -25 * (1 + mag.amax(-1, keepdim=True)) if self.q.dtype == torch.float16 else 0.0
        err = (self.out.double() - out).abs()
        bound = (u + 1e-4) * mag + u * out.abs() + 64 * small
        assert (err <= bound).all(), float((err / bound.clamp(min=1e-30)).max())
        empty = torch.isinf(lse)
        assert torch.equal(torch.isinf(self.lse), empty)
        assert ((self.lse.double() - lse).abs()[~empty] <= 2e-5).all()
        assert (self.out[empty] == 0).all()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,N", [(8, 2), (4, 4), (7, 1)])
@pytest.mark.parametrize("counts,lens,P", [
    ([1], [1], 0), ([1], [1], 1), ([1], [200], 63), ([1, 1, 1], [5, 64, 129], 65), ([1] * 9, range(1, 10), 600),
    ([3, 1, 5], [3, 70, 33], 130), ([2] * 17, [2 + 13 * i for i in range(17)], 300), ([40, 7], [40, 300], 77)])
def test_matches_formula(counts, lens, P, H, N, D, dt):
    c = Case(list(counts), lens, P, H, N, D, dt, seed=P + H)
    c.run()
    c.check()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts(dt, D):
    """Enough rows for the form that walks prefix and own keys in one workgroup."""
    c = Case([130, 1, 64, 300], [130, 90, 64, 301], 193, 128, 64, D, dt, seed=1)
    c.run()
    c.check()


@pytest.mark.parametrize("P", [0, 5])
@pytest.mark.parametrize("H,N,counts,lens", [(8, 2, [1, 2, 1, 4], [0, 1, -3, 2]), (64, 64, [300, 200], [3, 0])])
def test_rows_that_see_nothing(P, H, N, counts, lens):
    """Own lengths of zero, below zero and shorter than the queries: those rows see the prefix alone, or nothing."""
    c = Case(counts, lens, P, H, N, 64, torch.bfloat16, seed=2, S=8)
    c.run()
    c.check()
    if P == 0:
        assert (c.out[0] == 0).all() or lens[0] > 0


def test_empty_sequences_and_capped_lengths():
    c = Case([0, 2, 0, 0, 3, 0], [4, 5, 0, 9, 50, 2], 20, 4, 2, 128, torch.float16, seed=3, S=12)
    c.lens[4] = 12                                  # a length above max_len counts as max_len
    g = torch.Generator(device="cuda").manual_seed(33)
    c.k[4], c.v[4] = (torch.randn(c.k[4].shape, generator=g, device="cuda").to(torch.float16) for _ in range(2))
    c.run()
    c.check()


def test_no_starts_is_one_token_each():
    c = Case([1] * 6, [3, 1, 40, 7, 64, 65], 100, 8, 8, 64, torch.bfloat16, seed=4)
    c.run()
    want = c.out.clone()
    c.attn.starts = None
    c.out.fill_(NAN)
    c.run()
    assert torch.equal(c.out, want)


@pytest.mark.parametrize("counts,lens,P", [([1, 1], [60, 9], 150), ([400, 500], [400, 520], 100)])
def test_head_major_layout(counts, lens, P):
    c = Case(counts, lens, P, 64, 16, 128, torch.bfloat16, seed=5, head_major=True)
    c.run()
    c.check()


@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_flat_and_steep_scores(size):
    c = Case([4, 1], [90, 33], 257, 8, 2, 128, torch.float16, seed=6, scale=size / 128 ** 0.5)
    c.run()
    out, lse, mag = su.attn64(c.q, c.kp, c.vp, c.k, c.v, c.starts, c.lens, c.scale)
    # scores of up to 30 x 40: their fp32 rounding moves a probability by up to 1e-3
    assert ((c.out.double() - out).abs() <= (2.0 ** -11 + 2e-3) * mag + 2.0 ** -11 * out.abs() + 2e-6).all()
    assert ((c.lse.double() - lse).abs() <= 1e-6 * lse.abs() + 2e-5).all()


def test_prefix_beyond_32_bits():
    """Keys 16 MiB apart: the last lie past 4 GiB."""
    P, N, D, dt = 300, 2, 64, torch.bfloat16
    stride = 16 << 20
    store = torch.empty((P, stride // 2), dtype=dt, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(7)
    kp, vp = store[:, :N * D].view(P, N, D), store[:, 4096:4096 + N * D].view(P, N, D)
    kp.copy_(torch.randn((P, N, D), generator=g, device="cuda"))
    vp.copy_(torch.randn((P, N, D), generator=g, device="cuda"))
    c = Case([1, 2], [4, 9], P, 4, N, D, dt, seed=8, prefix=(kp, vp))
    c.run()
    c.check()


def test_steady_bits_other_stream_and_graph():
    c = Case([2, 1, 5], [64, 200, 31], 700, 16, 4, 128, torch.bfloat16, seed=9, S=256)
    for b, n in enumerate(c.lens):                 # lengths may change under the graph
        g = torch.Generator(device="cuda").manual_seed(90 + b)
        c.k[b, n:], c.v[b, n:] = (torch.randn(c.k[b, n:].shape, generator=g, device="cuda").to(c.k.dtype) for _ in range(2))
    c.run()
    want = c.out.clone(), c.lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.run()
    assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run(sync=False)
    for lens in ([64, 200, 31], [3, 256, 100], [2, 1, 5], [0, 17, 256]):
        c.dev_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.lens = lens
        c.out.fill_(NAN)
        g.replay()
        torch.cuda.synchronize()
        c.check()
        got = c.out.clone()
        c.run()
        assert torch.equal(c.out, got)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("counts,lens,P,H,N", [([5, 1, 3], [40, 7, 3], 70, 8, 2), ([2] * 10, [9] * 10, 64, 16, 4),
                                               ([130, 200], [130, 260], 100, 64, 32)])
def test_broken_values_reach_the_queries_that_see_them_only(counts, lens, P, H, N, dt):
    """Infinities and NaN in the keys and values of a sequence's later tokens leave its earlier queries alone."""
    c = Case(counts, lens, P, H, N, 128, dt, seed=12)
    whole = torch.ones(len(c.q), dtype=torch.bool, device="cuda")
    for b, (n, own) in enumerate(zip(counts, lens)):
        if n < 2:
            continue
        c.v[b, own - 1, :, 3], c.v[b, own - 1, :, 77], c.k[b, own - 1, 0, 9] = NAN, float("inf"), NAN
        whole[c.starts[b + 1] - 1] = False
    c.run()
    out, lse, mag = su.attn64(c.q, c.kp, c.vp, c.k, c.v, c.starts, c.lens, c.scale)
    u = su.U16[dt]
    err = (c.out.double() - out).abs()
    assert (err <= (u + 1e-4) * mag + u * out.abs() + 64 * 2.0 ** -25 * (1 + mag.amax(-1, keepdim=True)))[whole].all()
    assert ((c.lse.double() - lse).abs() <= 2e-5)[whole].all()
    assert torch.isnan(c.out[~whole][:, :, 3]).all() and not torch.isfinite(c.out[~whole][:, :, 77]).any()


@pytest.mark.parametrize("counts,lens", [([1, 1, 1], [300, 1, 1999]), ([5], [2500]), ([3] * 40, [700] * 39 + [3])])
def test_caches_with_more_room_than_keys(counts, lens):
    """Parts of the own keys follow the lengths, not the cache's room."""
    c = Case(counts, lens, 700, 8, 2, 128, torch.bfloat16, seed=21, S=9000)
    c.run()
    c.check()
    tight = Case(counts, lens, 700, 8, 2, 128, torch.bfloat16, seed=21)
    for name in ("q", "kp", "vp"):
        getattr(tight, name).copy_(getattr(c, name))
    tight.k.copy_(c.k[:, :max(lens)]), tight.v.copy_(c.v[:, :max(lens)])
    tight.run()
    tight.check()


@pytest.mark.parametrize("P", [1, 33, 300, 1000])
@pytest.mark.parametrize("counts", [[1, 1], [20, 9]])
def test_an_infinite_value_at_the_end_of_the_prefix(P, counts):
    """All rows see it: their outputs are that infinity in its channel and nothing else changes."""
    c = Case(counts, [40, 30], P, 4, 2, 64, torch.float16, seed=22)
    c.q.mul_(0.25)                                        # so that no probability vanishes
    want, _, mag = su.attn64(c.q, c.kp, c.vp, c.k, c.v, c.starts, c.lens, c.scale)
    c.vp[P - 1, :, 7] = float("inf")
    c.run()
    assert (c.out[..., 7] == float("inf")).all()
    u, rest = su.U16[torch.float16], torch.arange(64, device="cuda") != 7
    bound = (u + 1e-4) * mag + u * want.abs() + 2.0 ** -19 * (1 + mag.amax(-1, keepdim=True))
    assert ((c.out.double() - want).abs() <= bound)[..., rest].all()
