"""Serving requests that come and go: the weight passes of wsr.h, the norms of wsr_step.h and the operators of wsr_serve.h on a
small random-weight decoder (head norms, rotary positions, grouped-query attention over a paged cache, a gated MLP).

    python examples/paged_decode.py [--requests 24] [--tokens 40]

A step feeds up to 16 tokens, what one weight pass takes: one of every request that is under way, and as much of the prompts of
those that wait as fits.  Each request's keys lie in pages of one pool, taken when it needs them and given back when it is done;
it begins when there is a place for it and the pool has pages for its whole answer beside those that others may still take.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_12114_amd import wsr  # noqa: E402

HALF = torch.float16
MOST = 16                        # tokens of a step


class Model:
    def __init__(self, layers=2, d=512, heads=8, kv_heads=2, dim=64, ffn=1024, vocab=1003, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std=1.0, mean=0.0, to=HALF):
            return torch.empty(shape, device="cuda").normal_(mean, std, generator=g).to(to)

        self.d, self.heads, self.kv_heads, self.dim, self.ffn, self.vocab = d, heads, kv_heads, dim, ffn, vocab
        self.shapes = {"q": (heads * dim, d), "k": (kv_heads * dim, d), "v": (kv_heads * dim, d), "o": (d, heads * dim),
                       "g": (ffn, d), "u": (ffn, d), "d": (d, ffn)}
        self.embed, self.head = normal(vocab, d, to=torch.float32), normal(vocab, d, std=2.5 * d ** -0.5)
        self.norm = normal(d, std=0.1, mean=1.0)
        self.freqs = (1e4 ** (-torch.arange(dim // 2, dtype=torch.float64, device="cuda") * 2 / dim)).float()
        self.layers = []
        for _ in range(layers):
            layer = {p: normal(M, K, std=K ** -0.5) for p, (M, K) in self.shapes.items()}
            for n, size in (("before_attn", d), ("before_mlp", d), ("q_norm", dim), ("k_norm", dim)):
                layer[n] = normal(size, std=0.1, mean=1.0)
            self.layers.append(layer)


class Server:
    """A pool of pages, the requests that hold them, and the buffers and structures of a step."""

    def __init__(self, model: Model, seqs=8, pages=64, page_size=16, longest=256, alternatives=4):
        m = self.model = model
        self.seqs, self.page_size, self.row = seqs, page_size, -(-longest // page_size)
        self.free = list(range(pages))
        self.held: list[list[int]] = [[] for _ in range(seqs)]
        new = lambda *shape, to=HALF: torch.empty(shape, dtype=to, device="cuda")  # noqa: E731
        f32, i32 = torch.float32, torch.int32
        self.h, self.x = new(MOST, m.d, to=f32), new(MOST, m.d)
        self.y = {p: new(MOST, M, to=f32) for p, (M, _) in m.shapes.items()}
        self.q16, self.a, self.act = new(MOST, m.heads, m.dim), new(MOST, m.heads, m.dim), new(MOST, m.ffn)
        self.logits = new(MOST, m.vocab, to=f32)
        self.starts, self.lens = new(seqs + 1, to=i32), new(seqs, to=i32)
        self.table = torch.full((seqs, self.row), -1, dtype=i32, device="cuda")
        self.given = new(MOST, to=i32)
        self.logp, self.rank, self.entropy = new(MOST, to=f32), new(MOST, to=i32), new(MOST, to=f32)
        self.top, self.top_logp = new(MOST, alternatives, to=i32), new(MOST, alternatives, to=f32)
        self.k = [new(pages, page_size, m.kv_heads, m.dim) for _ in m.layers]
        self.v = [torch.empty_like(k) for k in self.k]
        key, sizes = 2 * m.kv_heads * m.dim, []
        inputs = {**{p: self.x for p in "qkvgu"}, "o": self.a, "d": self.act}

        def weights(name, w):
            mats = wsr.make_mats(dict(fmt=wsr.WSR_F16, M=w[p].shape[0], K=w[p].shape[1], w=w[p], x=inputs[p],
                                      x_tok_stride=2 * w[p].shape[1], y=self.y[p], y_tok_stride=4 * w[p].shape[0]) for p in name)
            sizes.append(wsr.wsr_sweep_workspace_bytes(mats))
            return mats

        def block(y, before):    # y into the residual stream, the next block's input out of it
            return wsr.make_block(kind=wsr.WSR_NORM_RMS, fmt=wsr.WSR_F16, d=m.d, y=y, y_tok_stride=4 * m.d, h=self.h,
                                  h_tok_stride=4 * m.d, h_out=self.h, h_out_tok_stride=4 * m.d, pre_w=before, x=self.x,
                                  x_tok_stride=2 * m.d)

        self.passes, self.append, self.attn = [], [], []
        self.blocks = [block(None, m.layers[0]["before_attn"])]
        for i, w in enumerate(m.layers):
            self.passes.append([weights(name, w) for name in ("qkv", "o", "gu", "d")])
            following = m.layers[i + 1]["before_attn"] if i + 1 < len(m.layers) else m.norm
            self.blocks += [block(self.y["o"], w["before_mlp"]), block(self.y["d"], following)]
            cache = wsr.make_pages(k=self.k[i], v=self.v[i], n_pages=pages, page_size=page_size, page_stride=key * page_size,
                                   tok_stride=key, head_stride=2 * m.dim, table=self.table, table_stride=4 * self.row, max_pages=self.row)
            self.append.append(wsr.make_qkv(
                fmt=wsr.WSR_F16, flags=wsr.WSR_QKV_NORM, kind=wsr.WSR_NORM_RMS, n_heads=m.heads, n_kv_heads=m.kv_heads,
                head_dim=m.dim, rot_dim=m.dim, n_seqs=seqs, q=self.y["q"], q_tok_stride=4 * m.heads * m.dim, k=self.y["k"],
                k_tok_stride=4 * m.kv_heads * m.dim, v=self.y["v"], v_tok_stride=4 * m.kv_heads * m.dim, q_w=w["q_norm"],
                k_w=w["k_norm"], freqs=m.freqs, starts=self.starts, lens=self.lens, q_out=self.q16,
                q_out_tok_stride=2 * m.heads * m.dim, q_out_head_stride=2 * m.dim, cache=cache))
            self.attn.append(wsr.make_paged(
                fmt=wsr.WSR_F16, n_heads=m.heads, n_kv_heads=m.kv_heads, head_dim=m.dim, n_seqs=seqs, n_tokens=MOST,
                scale=m.dim ** -0.5, max_len=self.row * page_size, q=self.q16, q_tok_stride=2 * m.heads * m.dim,
                q_head_stride=2 * m.dim, starts=self.starts, lens=self.lens, out=self.a, out_tok_stride=2 * m.heads * m.dim,
                out_head_stride=2 * m.dim, cache=cache))
            sizes.append(wsr.wsr_paged_workspace_bytes(self.attn[-1]))
        self.out = wsr.make_mats([dict(fmt=wsr.WSR_F16, M=m.vocab, K=m.d, w=m.head, x=self.x, x_tok_stride=2 * m.d, y=self.logits,
                                       y_tok_stride=4 * m.vocab)])
        self.scores = wsr.make_logprobs(n_rows=MOST, vocab=m.vocab, n_top=alternatives, logits=self.logits, row_stride=4 * m.vocab,
                                        tokens=self.given, logp=self.logp, rank=self.rank, entropy=self.entropy, top=self.top,
                                        top_logp=self.top_logp)
        sizes += [wsr.wsr_sweep_workspace_bytes(self.out), wsr.wsr_logprobs_workspace_bytes(self.scores)]
        self.ws = new(max(sizes), to=torch.uint8)

    def hold(self, seq: int, length: int) -> None:
        """Pages for `length` places of a sequence; all of them back where it is 0."""
        need = -(-length // self.page_size)
        while len(self.held[seq]) < need:
            self.held[seq].append(self.free.pop())
        while len(self.held[seq]) > need:
            self.free.append(self.held[seq].pop())

    def run(self, counts: list[int], lens: list[int], tokens: list[int], given: list[int], stream) -> None:
        """A step: counts[b] tokens of each sequence, the last of its lens[b] places; `given` are the tokens whose log
        probabilities are asked for, one per row."""
        T, ws, size = len(tokens), self.ws, self.ws.numel()
        for b, n in enumerate(lens):
            self.hold(b, n)
        rows = [r + [-1] * (self.row - len(r)) for r in self.held]
        self.table.copy_(torch.tensor(rows, dtype=torch.int32))
        self.starts.copy_(torch.tensor([sum(counts[:b]) for b in range(self.seqs + 1)], dtype=torch.int32))
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        self.given[:T].copy_(torch.tensor(given, dtype=torch.int32))
        torch.index_select(self.model.embed, 0, torch.tensor(tokens, device="cuda"), out=self.h[:T])
        for s in (*self.blocks, *self.append, *self.attn):
            s.n_tokens = T
        self.scores.n_rows = T

        def norm(i):
            wsr.wsr_block_norm(self.blocks[i], stream)

        norm(0)
        for i, (qkv, o, gu, d) in enumerate(self.passes):
            wsr.wsr_decode_sweep_mma(qkv, T, ws, size, stream)
            wsr.wsr_append_qkv(self.append[i], stream)
            wsr.wsr_paged_attention(self.attn[i], ws, size, stream)
            wsr.wsr_decode_sweep_mma(o, T, ws, size, stream)
            norm(2 * i + 1)
            wsr.wsr_decode_sweep_mma(gu, T, ws, size, stream)
            self.act[:T].copy_(torch.nn.functional.silu(self.y["g"][:T]) * self.y["u"][:T])
            wsr.wsr_decode_sweep_mma(d, T, ws, size, stream)
            norm(2 * i + 2)
        wsr.wsr_decode_sweep_mma(self.out, T, ws, size, stream)
        wsr.wsr_token_logprobs(self.scores, ws, size, stream)


def serve(server: Server, prompts: list[list[int]], n: int, each=None):
    """Greedy answers of n tokens to every prompt, in their order, as many at a time as there are places and pages for.
    Returns each prompt's tokens, its own log probability (of all but its first token) and the answer's.
    `each(requests, counts, tokens)` is called after every step."""
    if n < 1 or not all(prompts) or server.seqs > MOST:
        raise ValueError(f"prompts and answers have tokens, and a step has at most {MOST}, one of each place")
    pages = [-(-(len(p) + n - 1) // server.page_size) for p in prompts]       # the last token's key is never stored
    most, promised = len(server.free), 0
    if max(pages, default=0) > min(most, server.row):
        raise ValueError(f"a request of {max(pages)} pages, where the pool has {most} and a sequence {server.row}")
    stream, waiting = torch.cuda.current_stream(), list(range(len(prompts)))
    history, scored = [list(p) for p in prompts], [[0.0, 0.0] for _ in prompts]
    places: list[int | None] = [None] * server.seqs      # the request in each place, and what of it is cached
    cached = [0] * len(prompts)
    while waiting or any(r is not None for r in places):
        for b, r in enumerate(places):
            if r is None and waiting and promised + pages[waiting[0]] <= most:
                places[b] = waiting.pop(0)
                promised += pages[places[b]]
        active = [r for r in places if r is not None]
        counts, room = [0] * server.seqs, MOST - len(active)
        for b, r in enumerate(places):                    # one token of each, and what fits of the prompts
            if r is not None:
                more = min(room, len(history[r]) - cached[r] - 1)
                counts[b], room = 1 + more, room - more
        tokens, given, lens = [], [], [0] * server.seqs
        for b, r in enumerate(places):
            if r is not None:
                tokens += history[r][cached[r]:cached[r] + counts[b]]
                given += (history[r] + [-1])[cached[r] + 1:cached[r] + counts[b] + 1]
                lens[b] = cached[r] + counts[b]
        server.run(counts, lens, tokens, given, stream)
        if each:
            each(places, counts, tokens)
        logp, best, best_logp = server.logp.tolist(), server.top[:, 0].tolist(), server.top_logp[:, 0].tolist()
        at = 0
        for b, r in enumerate(places):
            if r is None:
                continue
            scored[r][0] += sum(v for v, x in zip(logp[at:at + counts[b]], given[at:at + counts[b]]) if x >= 0)
            at, cached[r] = at + counts[b], cached[r] + counts[b]
            if cached[r] == len(history[r]):              # all of it is cached: the last row's best is the next token
                history[r].append(best[at - 1])
                scored[r][1] += best_logp[at - 1]
                if len(history[r]) == len(prompts[r]) + n:
                    places[b] = None
                    server.hold(b, 0)
                    promised -= pages[r]
    return history, scored


def workload(requests: int, n: int):
    """Prompts, and the sizes of a server that answers them with n tokens each: five places' worth of pages for its eight."""
    prompts = [[(7 * i * i + r) % 61 for i in range(5 + 17 * r % 90)] for r in range(requests)]
    longest = max(map(len, prompts)) + n
    return prompts, dict(seqs=8, pages=5 * -(-longest // 16), page_size=16, longest=longest)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--requests", type=int, default=24)
    p.add_argument("--tokens", type=int, default=40)
    o = p.parse_args()
    prompts, sizes = workload(o.requests, o.tokens)
    server = Server(Model(), **sizes)
    serve(server, prompts[:2], min(2, o.tokens))
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    history, scored = serve(server, prompts, o.tokens)
    torch.cuda.synchronize()
    seconds, n = time.perf_counter() - t0, sum(map(len, history))
    print(f"{n} tokens of {o.requests} requests in {seconds:.3f} s; mean log probability of the answers' tokens "
          f"{sum(s[1] for s in scored) / (o.requests * o.tokens):.3f}; {len(server.free)} pages free")


if __name__ == "__main__":
    main()
