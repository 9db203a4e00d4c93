"""wsr_paged_attention of many sequences: up to the most a call takes, on both sides of the choice between waves that search
all of them and sums written once, and with starts that fall."""
import time

import pytest
import torch

import serve_util as su
from gpu_util import needs_gpu, stream
from paper_2608_12114_amd import wsr
from test_gpu_serve_paged import BF16, F16, Case

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("seqs", [191, 192, 193, 256, 512, 513, 1023, 1025, 4097])
@pytest.mark.parametrize("H,N", [(4, 1), (6, 3)])
@pytest.mark.parametrize("room", [0, 2000])
def test_counts_of_sequences(seqs, H, N, room):
    """Empty sequences, drafts and lengths of all kinds among them; a few are long enough to be cut where there is room."""
    counts = [(b % 7 == 0) * 4 + (b % 5 != 0) for b in range(seqs)]
    lens = [n + (13 * b) % 37 + (1500 if room and b % 97 == 3 else 0) for b, n in enumerate(counts)]
    c = Case(counts, lens, H, N, 64, BF16, page=8, room=room, first=2, after=1, seed=seqs)
    c.run()
    c.check()


@pytest.mark.parametrize("D,G,n", [(64, 4, 1), (128, 8, 3), (64, 8, 8), (256, 4, 7), (128, 8, 14), (64, 8, 30)])
def test_long_sequences_among_many(D, G, n):
    """Of 600 sequences one with 9000 keys and one with 2500, which are cut into parts, in tiles of each height."""
    counts = [n if b % 3 == 0 else 1 for b in range(600)]
    lens = [n + b % 11 for b, n in enumerate(counts)]
    lens[17], lens[599] = 9000, 2500
    c = Case(counts, lens, G, 1, D, F16, page=16, seed=n)
    c.run()
    c.check()


def test_same_bits_among_many():
    c = Case([1] * 700, [1 + 7 * b for b in range(700)], 8, 2, 64, BF16, page=32)
    c.run()
    first = c.out.clone(), c.lse.clone()
    c.check()
    for _ in range(3):
        c.out.fill_(77.0)
        c.run()
        assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])


@pytest.mark.parametrize("room", [0, 4000])
def test_as_many_as_a_call_takes(room):
    """2^20 sequences of no key, a hole, or one key, whose value is the result bit for bit; all of it well within a second:
    what a workgroup reads does not grow with the sequences (searched by each for its own, 2^20 x 2^20 / 64 loads, it would
    be seconds)."""
    B, D = 1 << 20, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(B, 1, D, generator=g, device="cuda").to(F16) for _ in range(3))
    page = 1 + room
    table = torch.randperm(B, generator=g, device="cuda").to(torch.int32)[:, None].contiguous()
    kind = torch.arange(B, device="cuda") % 5
    table[kind == 1] = -1
    lens = (kind != 0).to(torch.int32)
    out, lse = torch.full_like(q, 77.0), torch.full((B, 1), 77.0, device="cuda")
    # a page has room for `page` keys, of which only the first is ever seen: pages overlap behind it
    cache = wsr.make_pages(k=k, v=v, n_pages=B, page_size=page, page_stride=2 * D, tok_stride=0, head_stride=2 * D, table=table, table_stride=4,
                           max_pages=1)
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    p = wsr.make_paged(fmt=wsr.WSR_F16, n_heads=1, n_kv_heads=1, head_dim=D, n_seqs=B, n_tokens=B, scale=D ** -0.5, max_len=page, q=q,
                       q_tok_stride=2 * D, q_head_stride=2 * D, starts=starts, lens=lens, out=out, out_tok_stride=2 * D,
                       out_head_stride=2 * D, lse=lse, cache=cache)
    ws = torch.full((wsr.wsr_paged_workspace_bytes(p),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    wsr.wsr_paged_attention(p, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 1.0
    seen = (kind > 1)[:, None]
    at = table[:, 0].clamp(min=0).long()
    assert torch.equal(out, torch.where(seen[..., None], v[at], torch.zeros_like(v)))
    want = (q.double() * k[at].double()).sum(-1) * D ** -0.5
    # 64 products in fp32, and the logarithm of 1
    assert torch.isneginf(lse[~seen]).all() and ((lse.double() - want).abs()[seen] <= 20 * 2.0 ** -24 * (1 + want.abs()[seen]) +
                                                16 * 2.0 ** -24 * ((q * k[at]).double().abs().sum(-1) * D ** -0.5)[seen]).all()


@pytest.mark.parametrize("H,N,n", [(8, 2, 1), (64, 8, 6)])
@pytest.mark.parametrize("room", [0, 3000])
def test_anything_stays_inside(H, N, n, room):
    """Starts that fall, lengths and pages of any value among many sequences: nothing around the outputs is touched."""
    seqs, D = 700, 64
    c = Case([n] * seqs, [n + 20] * seqs, H, N, D, F16, page=24, room=room)
    c.k.fill_(0.5), c.v.fill_(0.25)
    g = torch.Generator().manual_seed(H + n)
    any32 = lambda t, lo=-2 ** 31, hi=2 ** 31 - 1: t.copy_(torch.randint(lo, hi, t.shape, generator=g))  # noqa: E731
    T, edge = n * seqs, 50
    wide, wide_lse = c.out.new_full((T + 2 * edge, H, D), 77.0), c.lse.new_full((T + 2 * edge, H), 77.0)
    need = wsr.wsr_paged_workspace_bytes(wsr.make_paged(**c.fields))
    ws = torch.full((need + (2 << 20),), 255, dtype=torch.uint8, device="cuda")
    for starts in ((-5, T + 5), (0, T + 1), (-2 ** 31, 2 ** 31 - 1), (T, T + 1)):
        any32(c.dev_starts, *starts), any32(c.dev_lens), any32(c.table)
        c.table[:, ::2] = torch.randint(0, c.k.shape[0], c.table[:, ::2].shape, generator=g).to(c.table)
        p = wsr.make_paged(**{**c.fields, "out": wide[edge:], "lse": wide_lse[edge:]})
        ws[need:] = 255
        wsr.wsr_paged_attention(p, ws, need, stream())
        torch.cuda.synchronize()
        for t in (wide, wide_lse):
            assert (t[:edge] == 77.0).all() and (t[T + edge:] == 77.0).all()
        assert (ws[need:] == 255).all()


def test_a_workspace_for_many_serves_fewer():
    """Of 300 sequences, which one launch serves, for 250, which take two and the sums."""
    c = Case([1] * 300, [1 + 3 * b for b in range(300)], 4, 1, 64, BF16, page=16, room=600)
    need = wsr.wsr_paged_workspace_bytes(wsr.make_paged(**{**c.fields, "starts": None}))
    ws = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    for seqs in (300, 250, 193, 192, 1):
        p = wsr.make_paged(**{**c.fields, "starts": None, "n_seqs": seqs, "n_tokens": seqs})
        assert wsr.wsr_paged_workspace_bytes(p) <= need
        c.out.fill_(77.0), c.lse.fill_(77.0)
        wsr.wsr_paged_attention(p, ws, need, stream())
        torch.cuda.synchronize()
        assert (c.out[seqs:] == 77.0).all() and (ws[need:] == 255).all()
        out, _, bound, _ = su.paged64(c.q[:seqs], c.k, c.v, c.table, c.page, list(range(seqs + 1)), c.lens[:seqs], c.max_len, c.scale)
        assert ((c.out[:seqs].double() - out).abs() <= bound).all()


def test_replayed_with_other_lengths():
    """A captured call of many sequences, replayed with other lengths and pages between eager calls: the eager call's bits."""
    c = Case([1] * 800, [1 + (37 * b) % 1500 for b in range(800)], 8, 2, 64, F16, page=16, room=1600)
    c.run()
    p, side = c.paged, torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        wsr.wsr_paged_attention(p, c.ws, c.ws.numel(), side)
    ws = torch.empty_like(c.ws)
    g = torch.Generator(device="cuda").manual_seed(3)
    c.k.nan_to_num_(0.25), c.v.nan_to_num_(0.5)
    for longest in (1500, 1, 90, 1600, 700):
        c.dev_lens.copy_(torch.randint(0, longest + 1, (800,), generator=g, device="cuda"))
        c.table.copy_(torch.randint(0, c.k.shape[0], c.table.shape, generator=g, device="cuda"))
        c.out.fill_(77.0), c.lse.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        got = c.out.clone(), c.lse.clone()
        c.out.fill_(78.0), c.lse.fill_(78.0)
        wsr.wsr_paged_attention(p, ws, ws.numel(), stream())
        torch.cuda.synchronize()
        assert torch.equal(c.out, got[0]) and torch.equal(c.lse, got[1])


def test_more_items_than_32_bits_hold():
    """Every other sequence from the first row to the last: their tiles together pass 2^31, and sums of them stay in range."""
    H, N, D, T, seqs = 64, 8, 64, 1 << 13, 1 << 19
    q = torch.zeros(T, H, D, dtype=F16, device="cuda")
    out, edge = torch.full((T + 2, H, D), 77.0, dtype=F16, device="cuda"), 1
    k = torch.ones(1, 4, N, D, dtype=F16, device="cuda")
    starts = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    starts[1::2] = T
    lens = torch.full((seqs,), 2, dtype=torch.int32, device="cuda")
    table = torch.zeros(seqs, 1, dtype=torch.int32, device="cuda")
    cache = wsr.make_pages(k=k, v=k, n_pages=1, page_size=4, page_stride=2 * k.stride(0), tok_stride=2 * N * D, head_stride=2 * D,
                           table=table, table_stride=4, max_pages=1)
    p = wsr.make_paged(fmt=wsr.WSR_F16, n_heads=H, n_kv_heads=N, head_dim=D, n_seqs=seqs, n_tokens=T, scale=1.0, max_len=4, q=q,
                       q_tok_stride=2 * H * D, q_head_stride=2 * D, starts=starts, lens=lens, out=out[edge:], out_tok_stride=2 * H * D,
                       out_head_stride=2 * D, cache=cache)
    ws = torch.empty(wsr.wsr_paged_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    wsr.wsr_paged_attention(p, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    assert (out[:edge] == 77.0).all() and (out[edge + T:] == 77.0).all()
    got = out[edge:edge + T]
    assert ((got == 0.0) | (got == 1.0)).all()
