"""The serving operators one after another: keys that were appended are the keys that attention reads, captured and replayed with
other lengths and pages, and calls on two streams at once."""
import pytest
import torch

import serve_util as su
from gpu_util import needs_gpu
from paper_2608_12114_amd import wsr

pytestmark = [pytest.mark.gpu, needs_gpu]
HALF = torch.bfloat16


class Step:
    """Queries, keys and values into a cache, attention over it, and scores of its output as if they were logits."""

    def __init__(self, seqs, H, N, D, page, row, seed=0, room=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g, self.dims, self.page, self.row, self.seqs = g, (H, N, D), page, row, seqs
        new = lambda *s, to=HALF: torch.zeros(s, dtype=to, device="cuda")  # noqa: E731
        f32, i32 = torch.float32, torch.int32
        self.pool = seqs * row + 2
        self.k, self.v = new(self.pool, page, N, D), new(self.pool, page, N, D)
        self.qkv = [new(seqs, h * D, to=f32) for h in (H, N, N)]
        self.q16, self.out, self.lse = new(seqs, H, D), new(seqs, H, D), new(seqs, H, to=f32)
        self.lens, self.table, self.tokens = new(seqs, to=i32), new(seqs, row, to=i32), new(seqs, to=i32)
        self.logits = new(seqs, H * D, to=f32)
        self.scores = [new(seqs, to=f32), new(seqs, to=i32), new(seqs, to=f32), new(seqs, 7, to=i32), new(seqs, 7, to=f32)]
        self.freqs = (1e4 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") * 2 / D)).float()
        cache = wsr.make_pages(k=self.k, v=self.v, n_pages=self.pool, page_size=page, page_stride=2 * page * N * D, tok_stride=2 * N * D,
                               head_stride=2 * D, table=self.table, table_stride=4 * row, max_pages=row)
        self.append = wsr.make_qkv(
            fmt=wsr.WSR_BF16, flags=wsr.WSR_QKV_NORM, n_heads=H, n_kv_heads=N, head_dim=D, rot_dim=D, n_seqs=seqs, n_tokens=seqs,
            q=self.qkv[0], q_tok_stride=4 * H * D, k=self.qkv[1], k_tok_stride=4 * N * D, v=self.qkv[2], v_tok_stride=4 * N * D,
            freqs=self.freqs, lens=self.lens, q_out=self.q16, q_out_tok_stride=2 * H * D, q_out_head_stride=2 * D, cache=cache)
        self.attn = wsr.make_paged(
            fmt=wsr.WSR_BF16, n_heads=H, n_kv_heads=N, head_dim=D, n_seqs=seqs, n_tokens=seqs, scale=D ** -0.5, max_len=row * page,
            q=self.q16, q_tok_stride=2 * H * D, q_head_stride=2 * D, lens=self.lens, out=self.out, out_tok_stride=2 * H * D,
            out_head_stride=2 * D, lse=self.lse, cache=cache)
        self.logp = wsr.make_logprobs(n_rows=seqs, vocab=H * D, n_top=7, logits=self.logits, row_stride=4 * H * D, tokens=self.tokens,
                                      logp=self.scores[0], rank=self.scores[1], entropy=self.scores[2], top=self.scores[3],
                                      top_logp=self.scores[4])
        self.ws = new(max(wsr.wsr_paged_workspace_bytes(self.attn), wsr.wsr_logprobs_workspace_bytes(self.logp)), to=torch.uint8)
        self.ws.fill_(255)

    def feed(self, lens):
        """Other inputs, lengths and pages, in place."""
        normal = lambda t: t.copy_(torch.randn(t.shape, generator=self.g, device="cuda"))  # noqa: E731
        for t in (*self.qkv, self.k, self.v):
            normal(t)
        self.lens.copy_(torch.tensor(lens))
        self.table.copy_(torch.randperm(self.pool, generator=self.g, device="cuda")[:self.seqs * self.row].view(self.seqs, self.row))
        self.tokens.copy_(torch.randint(0, self.logits.shape[1], (self.seqs,), generator=self.g, device="cuda"))

    def call(self, stream):
        wsr.wsr_append_qkv(self.append, stream)
        wsr.wsr_paged_attention(self.attn, self.ws, self.ws.numel(), stream)
        self.logits.copy_(self.out.view(self.seqs, -1))
        wsr.wsr_token_logprobs(self.logp, self.ws, self.ws.numel(), stream)

    def results(self):
        return [t.clone() for t in (self.q16, self.k, self.v, self.out, self.lse, *self.scores)]

    def check(self, lens, before):
        H, N, D = self.dims
        at = torch.tensor([[n - 1 for n in lens]], device="cuda")
        for x, h, slot in ((self.qkv[1], N, self.k), (self.qkv[0], H, None)):
            want, err = su.turned64(x.view(self.seqs, h, D), at, self.freqs, None, rot=D, pairs=False, kind="rms")
            for b, n in enumerate(lens):
                got = self.q16[b] if slot is None else slot[int(self.table[b, (n - 1) // self.page]), (n - 1) % self.page]
                assert ((got.double() - want[b]).abs() <= err[b] * 1.01 + 2.0 ** -8 * want[b].abs()).all()
        out, lse, bound, lbound = su.paged64(self.q16, self.k, self.v, self.table, self.page, list(range(self.seqs + 1)), lens,
                                             self.row * self.page, D ** -0.5)
        assert ((self.out.double() - out).abs() <= bound).all() and ((self.lse.double() - lse).abs() <= lbound).all()
        for b in range(self.seqs):
            logp, rank, entropy, top, top_logp = su.logprobs64(self.logits[b], int(self.tokens[b]), 1.0, 7)
            assert int(self.scores[1][b]) == rank and self.scores[3][b].tolist() == top
            assert abs(float(self.scores[0][b]) - logp) <= su.logp_bound(H * D, logp)
        changed = (self.k != before).any(-1).any(-1).sum()    # one slot a sequence, nothing else
        assert int(changed) == self.seqs


CASES = [(3, 8, 2, 128, 16, 40, [1, 600, 77], [13, 2, 640]), (5, 4, 4, 64, 7, 500, [3499, 1, 900, 20, 3500], [5, 3000, 2, 1, 64]),
         (70, 8, 1, 64, 16, 4, [1 + b % 60 for b in range(70)], [64 - b % 50 for b in range(70)])]


@pytest.mark.parametrize("seqs,H,N,D,page,row,lens,others", CASES)
def test_appended_keys_are_read(seqs, H, N, D, page, row, lens, others):
    s = Step(seqs, H, N, D, page, row)
    for n in (lens, others):
        s.feed(n)
        before = s.k.clone()
        s.call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        s.check(n, before)


@pytest.mark.parametrize("seqs,H,N,D,page,row,lens,others", CASES)
def test_replayed_with_other_lengths(seqs, H, N, D, page, row, lens, others):
    """A captured step, replayed with other inputs, lengths and pages between eager calls, gives the eager step's bits."""
    s, eager = Step(seqs, H, N, D, page, row, seed=1), Step(seqs, H, N, D, page, row, seed=1)
    for t in (s, eager):
        t.feed(lens)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    s.call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        s.call(stream)
    eager.call(torch.cuda.current_stream())
    for n in (lens, others, [max(1, v // 2) for v in lens], others, lens):
        for t in (s, eager):
            t.feed(n)
        graph.replay()
        torch.cuda.synchronize()
        got = s.results()
        eager.call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        for a, b in zip(got, eager.results()):
            assert torch.equal(a, b)
        graph.replay()                                        # again on what is there
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, s.results()))


def test_two_streams_at_once():
    """Steps with workspaces of their own on two streams beside each other give what they give alone."""
    steps = [Step(*c[:6], seed=i) for i, c in enumerate(CASES[:2])]
    for s, c in zip(steps, CASES):
        s.feed(c[6])
    streams = [torch.cuda.Stream() for _ in steps]
    alone = []
    for s in steps:
        s.call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        alone.append(s.results())
    for _ in range(10):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.call(st)
    torch.cuda.synchronize()
    for s, want in zip(steps, alone):
        assert all(torch.equal(a, b) for a, b in zip(s.results(), want))
