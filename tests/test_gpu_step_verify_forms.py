"""wsr_verify_drafts in both of its chunk lengths (2048 logits for few, 4096 for many), with one chunk, a few and thousands
of them per sequence: rules, ties across chunks, broken rows, steady bits."""
import pytest
import torch

from gpu_util import needs_gpu
from test_gpu_step_verify import INF, NAN, Case

pytestmark = [pytest.mark.gpu, needs_gpu]


def chunks_of(B, V):
    """(logits of a chunk, chunks of a sequence), by the launch's rule."""
    size = 2048 if B * -(-V // 4096) < 512 else 4096
    return size, -(-V // size)


@pytest.mark.parametrize("points", [False, True])
@pytest.mark.parametrize("B,n,V,form", [(15, 2, 128256, (2048, 63)), (16, 3, 128256, (4096, 32)), (63, 2, 32768, (2048, 16)),
                                        (64, 3, 32768, (4096, 8)), (57, 1, 32769, (4096, 9)), (171, 2, 8195, (4096, 3)), (512, 2, 4095, (4096, 1)),
                                        (260, 5, 4097, (4096, 2)), (2, 1, 300007, (2048, 147)), (5, 2, 420001, (4096, 103))])
def test_matches_rules(B, n, V, form, points):
    assert chunks_of(B, V) == form
    c = Case(B, n, V, seed=B + V, points=points, pad=3)
    c.run()
    c.check()


def test_the_largest_vocabulary():
    V = 1 << 24
    assert chunks_of(1, V) == (4096, 4096)
    c = Case(1, 1, V, seed=70)
    c.run()
    c.check(skip=1.0)
    c.target[:], c.uniform[:] = -5.0, 0.0                   # a lone largest logit at the end, reached greedily
    c.target[:, :, V - 1], c.tokens[:], c.temps[:] = 1.0, V - 1, 0.0
    c.run()
    assert c.out.tolist() == [[V - 1, V - 1]] and c.accepted.tolist() == [1] and (c.logp == 0).all()


def test_ties_across_long_chunks():
    """Equal logits and equal scores go to the lowest index, also where they lie in different chunks."""
    B, V = 72, 40000
    assert chunks_of(B, V) == (4096, 10)
    c = Case(B, 1, V, seed=71, temps=(0.0, 1.0))
    c.target[:], c.draft[:], c.noise[:], c.uniform[:] = 0.0, 0.0, 1.0, 0.0
    first = [b * 541 % 39000 for b in range(B)]
    for b, i in enumerate(first):
        c.target[b, :, i:V:4096 if b % 3 else 1] = 2.0
        c.draft[b, :, i] = 2.0 if b % 2 == 0 else 0.0
        c.tokens[b, 0] = i
    c.run()
    assert c.accepted.tolist() == [1] * B
    assert c.out.tolist() == [[i, i] for i in first]


def test_broken_rows_in_long_chunks():
    B, V = 70, 32003
    assert chunks_of(B, V) == (4096, 8)
    c = Case(B, 2, V, seed=72, temps=(1.0, 0.8), counts=[b % 3 for b in range(B)])
    c.target[0::7, :, ::2] = NAN                            # NaN counts as -inf
    c.target[1::7, 0] = -INF                                # nothing to draw
    c.target[2::7, 0], c.target[2::7, 0, 4096 * 5 + 77] = -INF, -3.0    # one token left
    c.target[3::7, 0, 5], c.target[3::7, 0, V - 1] = INF, INF           # they share everything
    c.target[4::7, 0] = torch.finfo(torch.float32).min      # all at the type's lowest value
    c.draft[5::7, 0] = -INF                                 # a draft without a distribution
    c.run()
    c.check(skip=0.1)


@pytest.mark.parametrize("B,n,V", [(3, 4, 128256), (66, 3, 32003)])
def test_steady_bits_and_graph(B, n, V):
    """The last workgroup of a sequence to finish joins its chunks, whichever it is; the counters start anew each time."""
    c = Case(B, n, V, seed=73)
    c.run()
    want = c.out.clone(), c.accepted.clone(), c.logp.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(3):
            c.run(sync=False)
    for k in range(5):
        c.out.fill_(-7), c.logp.fill_(NAN), c.accepted.fill_(-7)
        c.ws.fill_(255 if k % 2 else 1)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want[0]) and torch.equal(c.accepted, want[1])
        assert torch.equal(c.logp.view(torch.int32), want[2].view(torch.int32))
