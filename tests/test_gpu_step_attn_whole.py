"""wsr_prefix_attention in its whole form, which takes a row tile through the prefix and its own keys at once: the last
round of workgroups cut into 2 to 16 parts along the keys, rows that see nothing, infinities and NaN, lengths that change
under a captured graph.  Each case states the form that it means."""
import math

import pytest
import torch

import step_util as su
from gpu_util import needs_gpu
from test_gpu_step_attn import NAN, Case

pytestmark = [pytest.mark.gpu, needs_gpu]
INF = float("inf")


def parts_of(counts, H, N, P, room):
    """Parts that each unit of the last round is cut into (1: uncut), by the launch's rules; 0: the split form."""
    G, held = H // N, 512
    rows = sum(counts) * G
    if rows <= 64 or rows < 64 * len(counts) or N * (rows // 128) < held // 2:
        return 0
    rest = N * sum(-(-n * G // 128) for n in counts) % held
    return min(max(1, min(16, (P + room) // 256)), held // rest) if rest else 1


def expected(c):
    """out, lse and sum p |v| in 64 bits, a sequence's rows of a key head at a time."""
    T, H, D = c.q.shape
    N, P = c.k.shape[2], c.kp.shape[0]
    out = torch.zeros((T, H, D), dtype=torch.float64, device="cuda")
    mag, lse = torch.zeros_like(out), torch.full((T, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(c.counts):
        own, t0 = min(max(c.lens[b], 0), c.k.shape[1]), c.starts[b]
        see = P + own - n + 1 + torch.arange(n, device="cuda")         # keys that each query sees
        hidden = torch.arange(P + own, device="cuda") >= see.clamp(min=P)[:, None]
        some = ~hidden.all(-1)
        if n == 0 or P + own == 0:
            continue
        for g in range(N):
            hs = slice(g * H // N, (g + 1) * H // N)
            k = torch.cat([c.kp[:, g], c.k[b, :own, g]]).double().t().contiguous()
            v = torch.cat([c.vp[:, g], c.v[b, :own, g]]).double()
            s = (c.q[t0:t0 + n, hs].double() @ k) * c.scale             # (n, G, keys)
            s = s.masked_fill(hidden[:, None], -math.inf)
            top = s.amax(-1, keepdim=True).clamp(min=-1e300)
            p = torch.exp(s - top)
            l = p.sum(-1, keepdim=True)
            lse[t0:t0 + n, hs] = (top + torch.log(l))[..., 0]
            p = torch.where(some[:, None, None], p / l, 0.0)
            v = torch.nan_to_num(v, 0.0, 0.0, 0.0)                      # rows that see broken values are compared apart
            out[t0:t0 + n, hs], mag[t0:t0 + n, hs] = p @ v, p @ v.abs()
    return out, lse, mag


def check(c, rows=None):
    """`rows` of q (all) as Case.check does."""
    out, lse, mag = expected(c)
    rows = torch.ones(len(c.q), dtype=torch.bool, device="cuda") if rows is None else rows
    u = su.U16[c.q.dtype]
    small = 2.0 ** -25 * (1 + mag.amax(-1, keepdim=True)) if c.q.dtype == torch.float16 else 0.0
    bound = (u + 1e-4) * mag + u * out.abs() + 64 * small
    err = (c.out.double() - out).abs()
    assert (err <= bound)[rows].all(), float((err / bound.clamp(min=1e-30))[rows].max())
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(c.lse)[rows], empty[rows])
    assert ((c.lse.double() - lse).abs() <= 2e-5)[rows & ~empty.any(-1)].all()
    assert (c.out[empty] == 0).all()


#        counts, lens, P, room, H, N, parts
CUT = [([130], [130], 400, 200, 384, 384, 2),
       ([200, 3], [260, 40], 333, 700, 300, 300, 1),
       ([130], [777], 65, 900, 300, 300, 3),
       ([129, 127], [129, 600], 800, 700, 172, 172, 5),
       ([257], [257], 1200, 300, 180, 180, 5),
       ([131], [1500], 2700, 1500, 260, 260, 16),
       ([140], [140], 0, 4100, 257, 257, 16),
       ([1037], [1037], 3100, 1037, 64, 8, 16),
       ([300, 0, 700, 41], [400, 9, 700, 50], 1000, 720, 64, 8, 6)]


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("counts,lens,P,room,H,N,parts", CUT)
def test_cut_last_round(counts, lens, P, room, H, N, parts, D, dt):
    assert parts_of(counts, H, N, P, room) == parts
    c = Case(counts, lens, P, H, N, D, dt, seed=P + N, S=room)
    c.run()
    check(c)


@pytest.mark.parametrize("P", [0, 5, 700])
@pytest.mark.parametrize("counts,lens,room,H,N,parts", [([300, 300], [3, 0], 8, 64, 64, 1), ([130, 130], [50, -4], 8, 150, 150, 1),
                                                        ([130, 200], [50, -4], 900, 130, 130, 3)])
def test_rows_that_see_nothing(counts, lens, room, H, N, parts, P):
    """Own lengths shorter than the queries, zero and below: those rows see the prefix alone, or nothing."""
    assert parts_of(counts, H, N, P, room) >= parts
    c = Case(counts, lens, P, H, N, 64, torch.bfloat16, seed=2, S=room)
    c.run()
    check(c)
    if P == 0:
        assert (c.out[0] == 0).all() and (c.lse[0] == -INF).all()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("counts,lens,P,room,H,N,parts", [([300, 300], [300, 340], 100, 340, 64, 64, 1), ([130], [777], 65, 900, 300, 300, 3),
                                                          ([257], [257], 1200, 300, 180, 180, 5), ([140], [140], 0, 4100, 257, 257, 16)])
def test_broken_values_reach_the_queries_that_see_them_only(counts, lens, P, room, H, N, parts, dt):
    """Infinities and NaN in the keys and values of each sequence's last token, and an infinite value in the middle of its
    own keys, which its first queries do not see."""
    assert parts_of(counts, H, N, P, room) == parts
    c = Case(counts, lens, P, H, N, 128, dt, seed=12, S=room)
    c.q.mul_(0.25)                                        # so that no probability vanishes
    last = torch.zeros(len(c.q), dtype=torch.bool, device="cuda")
    middle = last.clone()
    for b, (n, own) in enumerate(zip(counts, lens)):
        c.v[b, own - 1, :, 3], c.v[b, own - 1, :, 77], c.k[b, own - 1, 0, 9] = NAN, INF, NAN
        c.v[b, own - n // 2, :, 5] = INF
        last[c.starts[b + 1] - 1] = True
        middle[c.starts[b + 1] - n // 2:c.starts[b + 1]] = True
    c.run()
    check(c, ~last & ~middle)
    rest = torch.arange(128, device="cuda") != 5
    between = middle & ~last
    assert (c.out[between][..., 5] == INF).all()
    for b, (n, own) in enumerate(zip(counts, lens)):
        c.v[b, own - n // 2, :, 5] = 0.0
    out, lse, mag = expected(c)
    u = su.U16[dt]
    bound = (u + 1e-4) * mag + u * out.abs() + 64 * 2.0 ** -25 * (1 + mag.amax(-1, keepdim=True))
    assert ((c.out.double() - out).abs() <= bound)[between][..., rest].all()
    assert ((c.lse.double() - lse).abs() <= 2e-5)[between].all()
    assert torch.isnan(c.out[last][..., 3]).all() and not torch.isfinite(c.out[last][..., 77]).any()


@pytest.mark.parametrize("counts,lens,P,room,H,N,parts", [([130], [777], 65, 900, 300, 300, 3), ([1037], [1037], 3100, 1037, 64, 8, 16)])
def test_steady_bits_and_graph(counts, lens, P, room, H, N, parts):
    assert parts_of(counts, H, N, P, room) == parts
    c = Case(counts, lens, P, H, N, 128, torch.bfloat16, seed=9, S=room)
    g = torch.Generator(device="cuda").manual_seed(90)
    for t in (c.k, c.v):                                  # lengths change under the graph
        t[0, lens[0]:] = torch.randn(t[0, lens[0]:].shape, generator=g, device="cuda").to(t.dtype)
    c.run()
    want = c.out.clone(), c.lse.clone()
    c.out.fill_(NAN)
    c.run()
    assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(sync=False)
    for n in (lens[0], 3, room, 0):
        c.dev_lens.fill_(n)
        c.lens = [n]
        c.out.fill_(NAN), c.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check(c)
        got = c.out.clone()
        c.run()
        assert torch.equal(c.out, got)
