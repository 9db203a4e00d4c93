"""What happens between the weight passes of a batched decode step, as measurable cases: the adapters
of many requests beside the shared projections, attention over a prefix that the batch shares, the
norms around a block with its gate and residual scale, and the verification of drafted tokens, each
through the entry points of paper_2608_12114_amd.wsr (`own`) or in plain torch operations.

Sizes are those of the 8B- and 70B-shaped models this library sweeps (widths 4096 and 8192, 32 or 64
heads of 128 over 8 key heads, ffn 14336, vocabulary 128256) and odd ones beside them.  Inputs come from
torch's seeded generator; how long and how many things are follows from the case alone."""
import math
import random

import torch

own = False
EPS = 1e-5


def listed():
    return [
        # one token's attention output back into the residual stream, 8B width: latency alone
        {"name": "norm_rms_1x4096", "op": "norm", "kind": "rms", "fmt": "bf16", "tokens": 1, "d": 4096, "post": True,
         "gate": "channel"},
        # the 16 tokens of one matrix-core pass, 70B width
        {"name": "norm_rms_16x8192", "op": "norm", "kind": "rms", "fmt": "f16", "tokens": 16, "d": 8192, "post": True,
         "gate": "none"},
        # a prompt, an odd count of tokens, layer norms with biases and a gate of each token's own
        {"name": "norm_layer_4099x8192", "op": "norm", "kind": "layer", "fmt": "bf16", "tokens": 4099, "d": 8192,
         "post": True, "gate": "token"},
        # a single request with an adapter on one projection: the smallest call
        {"name": "lora_1tok_4096x4096_r16", "op": "lora", "fmt": "bf16", "tokens": 1, "layers": 1, "shapes": "o",
         "d": 4096, "kv": 1024, "ffn": 14336, "rank": 16, "adapters": 4},
        # 16 requests of 16 adapters over every projection of the 8B model, one sweep
        {"name": "lora_16tok_8b_r16", "op": "lora", "fmt": "f16", "tokens": 16, "layers": 32, "shapes": "qkvogud",
         "d": 4096, "kv": 1024, "ffn": 14336, "rank": 16, "adapters": 14},
        # prompts of six requests, five adapters of up to 64 ranks, the gate and up projections
        {"name": "lora_2055tok_ffn_r64", "op": "lora", "fmt": "bf16", "tokens": 2055, "layers": 1, "shapes": "gu",
         "d": 4096, "kv": 1024, "ffn": 14336, "rank": 64, "adapters": 5},
        # four sequences decode behind a short system prompt
        {"name": "attn_4seq_p1024", "op": "attn", "fmt": "f16", "seqs": 4, "queries": 1, "prefix": 1024, "own": 200,
         "heads": 32, "kv_heads": 8, "dim": 128},
        # 24 sequences, four drafts and the last token each, behind a long document, 70B heads
        {"name": "attn_24seq_5q_p32771", "op": "attn", "fmt": "bf16", "seqs": 24, "queries": 5, "prefix": 32771,
         "own": 1500, "heads": 64, "kv_heads": 8, "dim": 128},
        # four new prompts behind a shared one
        {"name": "attn_4seq_900q_p8192", "op": "attn", "fmt": "bf16", "seqs": 4, "queries": 900, "prefix": 8192,
         "own": 900, "heads": 32, "kv_heads": 8, "dim": 128},
        # one sequence, four drafts with their distributions, the whole vocabulary
        {"name": "verify_1seq_4d_128256", "op": "verify", "seqs": 1, "drafts": 4, "vocab": 128256, "points": False},
        # tokens looked up, not drawn (no draft distribution), an odd vocabulary
        {"name": "verify_5seq_2d_32003_points", "op": "verify", "seqs": 5, "drafts": 2, "vocab": 32003, "points": True},
        # a serving batch of 64 sequences with seven drafts each
        {"name": "verify_64seq_7d_128256", "op": "verify", "seqs": 64, "drafts": 7, "vocab": 128256, "points": False},
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _odd(rng, lo, hi):
    return min(int(_log(rng, lo, hi + 1)) | 1, hi)


def draw(rng):
    op = rng.choice(("norm", "lora", "attn", "verify"))
    if op == "norm":
        d = rng.choice((2048, 4096, 8192, 14336, 8 * _odd(rng, 16, 2047)))
        return {"op": op, "kind": rng.choice(("rms", "layer")), "fmt": rng.choice(("f16", "bf16")),
                "tokens": min(_odd(rng, 1, 8193), 4099 * 8192 // d), "d": d, "post": rng.random() < 0.75,
                "gate": rng.choice(("none", "channel", "token"))}
    if op == "lora":
        d, kv, ffn = rng.choice(((4096, 1024, 14336), (8192, 1024, 28672), (2048, 512, 5632), (1160, 392, 3976)))
        tokens, rank = _odd(rng, 1, 1025), rng.choice((4, 8, 16, 16, 24, 32, 64))
        adapters, shapes = max(1, min(tokens, int(_log(rng, 1, 33)))), rng.choice(("o", "qv", "qkvo", "gud", "qkvogud"))
        case = {"op": op, "fmt": rng.choice(("f16", "bf16")), "tokens": tokens, "layers": 1, "shapes": shapes, "d": d,
                "kv": kv, "ffn": ffn, "rank": rank, "adapters": adapters}
        most = int(1.2e9 / work(case)["bytes"])
        return dict(case, layers=max(1, min(32, most, int(_log(rng, 1, 33)))))
    if op == "attn":
        heads, kv = rng.choice(((32, 8), (64, 8), (32, 32), (12, 4), (7, 1)))
        queries = rng.choice((1, 1, 1, _odd(rng, 2, 16), _odd(rng, 17, 700)))
        seqs = rng.choice((1, _odd(rng, 2, 64))) if queries < 17 else rng.randint(1, 4)
        return {"op": op, "fmt": rng.choice(("f16", "bf16")), "seqs": seqs, "queries": queries,
                "prefix": _odd(rng, 1, 32771 if queries < 17 else 8191), "own": queries + _odd(rng, 1, 1500 if seqs < 33 else 700),
                "heads": heads, "kv_heads": kv, "dim": rng.choice((64, 128, 128))}
    return {"op": op, "seqs": _odd(rng, 1, 63), "drafts": rng.randint(1, 7), "vocab": rng.choice((128256, 32000, _odd(rng, 1001, 151937))),
            "points": rng.random() < 0.3}


# ---- what follows from the case alone ----------------------------------------------------------------

def _half(case):
    return torch.bfloat16 if case["fmt"] == "bf16" else torch.float16


def _projections(case):
    """[(M, K)] of the projections that have adapters, layer after layer."""
    d, kv, ffn = case["d"], case["kv"], case["ffn"]
    shape = {"q": (d, d), "k": (kv, d), "v": (kv, d), "o": (d, d), "g": (ffn, d), "u": (ffn, d), "d": (d, ffn)}
    return [shape[s] for s in case["shapes"]] * case["layers"]


def _tokens_with(case):
    """Tokens that have an adapter: one in eight has none, where there are enough of them."""
    return case["tokens"] - case["tokens"] // 8


def _ranks(case):
    """Each adapter's rank: every third has half, where all of them are used."""
    n, r = case["adapters"], case["rank"]
    return [r // 2 if a % 3 == 2 and _tokens_with(case) >= n else r for a in range(n)]


def _lengths(case):
    """[(queries, own keys)] of each sequence: the first is as long as the case says."""
    r, out = random.Random(7919 * case["seqs"] + case["own"]), [(case["queries"], case["own"])]
    for _ in range(case["seqs"] - 1):
        n = case["queries"] if case["queries"] < 17 else r.randint(case["queries"] // 4, case["queries"])
        out.append((n, r.randint(n, max(n, case["own"]))))
    return out


# ---- inputs, from the seed alone -----------------------------------------------------------------------

def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, to=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(to)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    if case["op"] == "norm":
        T, d, h = case["tokens"], case["d"], _half(case)
        spread = torch.exp(normal(d, std=0.7))            # channels differ in size, as in a trained model
        s = {"y": normal(T, d) * spread, "h": normal(T, d, std=3.0) * spread, "pre_w": normal(d, std=0.2, mean=1.0, to=h)}
        if case["post"]:
            s["post_w"] = normal(d, std=0.2, mean=1.0, to=h)
        if case["kind"] == "layer":
            s["pre_b"] = normal(d, std=0.1, to=h)
            if case["post"]:
                s["post_b"] = normal(d, std=0.1, to=h)
        if case["gate"] != "none":
            s["gate"] = normal(*((T, d) if case["gate"] == "token" else (1, d)), std=0.3, mean=0.5, to=h)
        return s
    if case["op"] == "lora":
        T, n, r, h = case["tokens"], case["adapters"], case["rank"], _half(case)
        perm = torch.randperm(n, device="cuda", generator=g)
        ids = torch.arange(T, device="cuda")
        whose = ids * n // _tokens_with(case) if T > 64 else ids % n
        ids = torch.where(ids < _tokens_with(case), perm[whose.clamp(max=n - 1)], -1)
        if T <= 64:                                        # decode: requests in any order; prompts: whole
            ids = ids[torch.randperm(T, device="cuda", generator=g)]
        sizes = [T * M for M, _ in _projections(case)]     # all outputs lie in one tensor, projection after projection
        flat = torch.zeros(sum(sizes), dtype=torch.float32, device="cuda")
        mods = [{"a": normal(n, r, K, std=K ** -0.5, to=h), "b": normal(n, M, r, std=0.02, to=h), "x": normal(T, K, to=h),
                 "y0": normal(T, M), "y": y.view(T, M)} for (M, K), y in zip(_projections(case), flat.split(sizes))]
        return {"mods": mods, "y": flat, "ids": ids.to(torch.int32), "ranks": ints(_ranks(case)),
                "scales": 16.0 / ints(_ranks(case)).float()}
    if case["op"] == "attn":
        H, N, D, h, per = case["heads"], case["kv_heads"], case["dim"], _half(case), _lengths(case)
        starts = [sum(q for q, _ in per[:i]) for i in range(len(per) + 1)]
        most = max(k for _, k in per)
        return {"q": normal(starts[-1], H, D, std=2.5, to=h), "k_prefix": normal(case["prefix"], N, D, to=h),
                "v_prefix": normal(case["prefix"], N, D, to=h), "k": normal(len(per), most, N, D, to=h),
                "v": normal(len(per), most, N, D, to=h), "starts": ints(starts), "lens": ints([k for _, k in per])}
    B, n, V = case["seqs"], case["drafts"], case["vocab"]
    target = normal(B, n + 1, V, std=2.5)
    draft = target[:, :n] + normal(B, n, V, std=0.6)
    heat = torch.tensor([(1.0, 0.7, 0.9, 0.0)[b % 4] for b in range(B)], dtype=torch.float32, device="cuda")
    pick = (draft - heat[:, None, None] * torch.empty_like(draft).exponential_(generator=g).log_()).argmax(-1)
    s = {"target": target, "draft": None if case["points"] else draft, "tokens": pick.to(torch.int32),
         "counts": ints([n - (b % 4 == 3) for b in range(B)]), "temperature": heat,
         "uniform": torch.rand((B, n), dtype=torch.float32, device="cuda", generator=g),
         "noise": torch.empty((B, V), dtype=torch.float32, device="cuda").exponential_(generator=g).clamp_(min=1e-30)}
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:                      # the tables and the workspace that a program keeps beside its buffers
        from paper_2608_12114_amd import wsr
        _handles(wsr, s, case)
    return s


def _handles(wsr, s, case):
    code = wsr.WSR_BF16 if case.get("fmt") == "bf16" else wsr.WSR_F16
    byte = torch.uint8
    if case["op"] == "norm":
        T, d = case["tokens"], case["d"]
        s["h_out"], s["x"] = torch.empty_like(s["h"]), torch.empty((T, d), dtype=_half(case), device="cuda")
        s["block"] = wsr.make_block(
            kind=wsr.WSR_NORM_RMS if case["kind"] == "rms" else wsr.WSR_NORM_LAYER, fmt=code, n_tokens=T, d=d,
            flags=wsr.WSR_BLOCK_POST if case["post"] else 0, y=s["y"], y_tok_stride=4 * d, post_w=s.get("post_w"),
            post_b=s.get("post_b"), gate=s.get("gate"), gate_tok_stride=2 * d if case["gate"] == "token" else 0,
            res_scale=0.9, h=s["h"], h_tok_stride=4 * d, h_out=s["h_out"], h_out_tok_stride=4 * d, pre_w=s["pre_w"],
            pre_b=s.get("pre_b"), x=s["x"], x_tok_stride=2 * d, eps=EPS)
    elif case["op"] == "lora":
        n, r = case["adapters"], case["rank"]
        s["table"] = wsr.make_loras(
            dict(fmt=code, rank=r, M=M, K=K, a=m["a"], a_stride=2 * r * K, b=m["b"], b_stride=2 * M * r, x=m["x"],
                 x_tok_stride=2 * K, y0=m["y0"], y0_tok_stride=4 * M, y=m["y"], y_tok_stride=4 * M)
            for (M, K), m in zip(_projections(case), s["mods"]))
        s["ws"] = torch.empty(wsr.wsr_lora_workspace_bytes(s["table"], case["tokens"]), dtype=byte, device="cuda")
    elif case["op"] == "attn":
        H, N, D = case["heads"], case["kv_heads"], case["dim"]
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
        s["attn"] = wsr.make_attn(
            fmt=code, n_heads=H, n_kv_heads=N, head_dim=D, n_seqs=case["seqs"], n_tokens=s["q"].shape[0],
            max_len=s["k"].shape[1], scale=D ** -0.5, q=s["q"], q_tok_stride=2 * H * D, q_head_stride=2 * D,
            k_prefix=s["k_prefix"], v_prefix=s["v_prefix"], prefix_len=case["prefix"], prefix_tok_stride=2 * N * D,
            prefix_head_stride=2 * D, k=s["k"], v=s["v"], kv_seq_stride=2 * N * D * s["k"].shape[1],
            kv_tok_stride=2 * N * D, kv_head_stride=2 * D, starts=s["starts"], lens=s["lens"], out=s["out"],
            out_tok_stride=2 * H * D, out_head_stride=2 * D, lse=s["lse"])
        s["ws"] = torch.empty(wsr.wsr_attn_workspace_bytes(s["attn"]), dtype=byte, device="cuda")
    else:
        B, n, V = case["seqs"], case["drafts"], case["vocab"]
        new = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        s["out"], s["accepted"], s["logp"] = new(B, n + 1), new(B), new(B, n + 1, dtype=torch.float32)
        s["verify"] = wsr.make_verify(
            n_seqs=B, n_drafts=n, vocab=V, target=s["target"], target_seq_stride=4 * V * (n + 1), target_row_stride=4 * V,
            draft=s["draft"], draft_seq_stride=4 * V * n, draft_row_stride=4 * V, tokens=s["tokens"], counts=s["counts"],
            temperature=s["temperature"], uniform=s["uniform"], noise=s["noise"], noise_seq_stride=4 * V, out=s["out"],
            accepted=s["accepted"], logp=s["logp"])
        s["ws"] = torch.empty(wsr.wsr_verify_workspace_bytes(s["verify"]), dtype=byte, device="cuda")


# ---- the measured calls --------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"norm": _norm, "lora": _lora, "attn": _attn, "verify": _verify}[op](s)
    from paper_2608_12114_amd import wsr
    stream = torch.cuda.current_stream()
    if op == "norm":
        wsr.wsr_block_norm(s["block"], stream)
        return {"h": s["h_out"], "x": s["x"]}
    if op == "lora":
        wsr.wsr_lora_sweep(s["table"], s["case"]["tokens"], s["ids"], s["case"]["adapters"], s["ranks"], s["scales"], s["ws"],
                           s["ws"].numel(), stream)
        return s["y"]
    if op == "attn":
        wsr.wsr_prefix_attention(s["attn"], s["ws"], s["ws"].numel(), stream)
        return {"out": s["out"], "lse": s["lse"]}
    wsr.wsr_verify_drafts(s["verify"], s["ws"], s["ws"].numel(), stream)
    return {"out": s["out"], "accepted": s["accepted"], "logp": s["logp"]}


def _normed(v, kind, w, b):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    v = v if w is None else v * w.float()
    return v if b is None else v + b.float()


def _norm(s):
    c, v = s["case"], s["y"]
    if c["post"]:
        v = _normed(v, c["kind"], s["post_w"], s.get("post_b"))
    if "gate" in s:
        v = v * s["gate"].float()
    h = 0.9 * s["h"] + v
    return {"h": h, "x": _normed(h, c["kind"], s["pre_w"], s.get("pre_b")).to(_half(c))}


def _lora(s):
    c = s["case"]
    n, r = c["adapters"], c["rank"]
    ids, rank = s["ids"][:, None, None], torch.arange(r, device="cuda")
    mine = (ids == torch.arange(n, device="cuda")[:, None]) & (rank < s["ranks"][:, None])
    weight = (mine.float() * s["scales"][:, None]).reshape(-1, n * r)

    def one(m):
        v = m["x"].float() @ m["a"].reshape(n * r, -1).float().t()
        torch.add(m["y0"], (v * weight) @ m["b"].transpose(1, 2).reshape(n * r, -1).float(), out=m["y"])

    [one(m) for m in s["mods"]]
    return s["y"]


def _attn(s):
    c, q = s["case"], s["q"].float()
    T, H, D = q.shape
    N = c["kv_heads"]
    G, S = H // N, s["k"].shape[1]
    first, lens = s["starts"][:-1].long(), s["lens"].long()
    counts = s["starts"][1:].long() - first
    q = q.reshape(T, N, G, D) * D ** -0.5
    # the shared keys, all sequences' queries at once
    kp, vp = s["k_prefix"].float().permute(1, 2, 0), s["v_prefix"].float().transpose(0, 1)
    a = q.transpose(0, 1).reshape(N, T * G, D) @ kp
    ma = a.amax(-1, keepdim=True)
    a = torch.exp(a - ma)
    la, oa = a.sum(-1, keepdim=True), a @ vp
    back = lambda v: v.reshape(N, T, G, -1).transpose(0, 1)  # noqa: E731
    ma, la, oa = back(ma), back(la), back(oa)
    # each sequence's own keys, queries padded to the longest sequence's
    most = c["queries"]
    i = torch.arange(most, device="cuda")
    at = (first[:, None] + i).clamp(max=T - 1)
    qo = q[at].transpose(1, 2).reshape(c["seqs"], N, most * G, D)
    ko, vo = s["k"].float().permute(0, 2, 3, 1), s["v"].float().transpose(1, 2)
    b = (qo @ ko).reshape(c["seqs"], N, most, G, S)
    seen = torch.arange(S, device="cuda") < (lens - counts)[:, None, None] + i[:, None] + 1
    b = b.masked_fill(~seen[:, None, :, None], -math.inf)
    mb = b.amax(-1, keepdim=True)
    b = torch.exp(b - mb.clamp(min=-3e38))
    lb = b.sum(-1, keepdim=True)
    ob = (b.reshape(c["seqs"], N, most * G, S) @ vo).reshape(c["seqs"], N, most, G, D)
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device="cuda"), counts, output_size=T)
    j = torch.arange(T, device="cuda") - first[seq]
    mb, lb, ob = mb[seq, :, j], lb[seq, :, j], ob[seq, :, j]
    m = torch.maximum(ma, mb)
    wa, wb = torch.exp(ma - m), torch.exp(mb - m)
    l = la * wa + lb * wb
    return {"out": ((oa * wa + ob * wb) / l).reshape(T, H, D).to(s["q"].dtype), "lse": (m + torch.log(l)).reshape(T, H)}


def _probabilities(logits, temperature, greedy):
    """Softmax at each sequence's temperature; at zero all of it is on the largest logit."""
    v = logits / torch.where(greedy, 1.0, temperature)[:, None, None]
    v = torch.exp(v - v.amax(-1, keepdim=True))
    p = v / v.sum(-1, keepdim=True)
    top = torch.zeros_like(p).scatter_(-1, logits.argmax(-1, keepdim=True), 1.0)
    return torch.where(greedy[:, None, None], top, p)


def _verify(s):
    c = s["case"]
    B, n = c["seqs"], c["drafts"]
    greedy = s["temperature"] == 0
    p = _probabilities(s["target"], s["temperature"], greedy)
    pick = s["tokens"].long()[..., None]
    if s["draft"] is None:
        q = torch.zeros_like(p[:, :n]).scatter_(-1, pick, 1.0)
    else:
        q = _probabilities(s["draft"], s["temperature"], greedy)
    px, qx = p[:, :n].gather(-1, pick)[..., 0], q.gather(-1, pick)[..., 0]
    place = torch.arange(n + 1, device="cuda")
    passed = (s["uniform"] * qx < px) & (place[:n] < s["counts"][:, None])
    accepted = passed.int().cumprod(-1).sum(-1)
    b = torch.arange(B, device="cuda")
    row = p[b, accepted]
    left = torch.where((accepted < s["counts"])[:, None], (row - q[b, accepted.clamp(max=n - 1)]).clamp(min=0), row)
    left = torch.where((left.amax(-1) > 0)[:, None], left, row)
    token = (left / s["noise"]).argmax(-1)
    at = place[None] - accepted[:, None]
    out = torch.cat([s["tokens"], s["tokens"][:, :1]], 1).long()
    out = torch.where(at < 0, out, torch.where(at == 0, token[:, None], -1))
    logp = torch.log(p.gather(-1, out.clamp(min=0)[..., None])[..., 0])
    return {"out": out.int(), "accepted": accepted.int(), "logp": torch.where(at <= 0, logp, 0.0)}


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    if case["op"] == "norm":
        T, d = case["tokens"], case["d"]
        gate = {"none": 0, "channel": 1, "token": T}[case["gate"]]
        rows = (1 + case["post"]) * (2 if case["kind"] == "layer" else 1)
        return {"bytes": T * d * (4 + 4 + 4 + 2) + 2 * d * (rows + gate), "flops": 12 * T * d}
    if case["op"] == "lora":
        T, used = case["tokens"], min(case["adapters"], _tokens_with(case))
        ranks = _ranks(case)
        if used < len(ranks):
            ranks = ranks[:used]
        per = -(-_tokens_with(case) // used)
        return {"bytes": sum(2 * sum(ranks) * (M + K) + T * (2 * K + 8 * M) for M, K in _projections(case)),
                "flops": sum(2 * per * sum(ranks) * (M + K) for M, K in _projections(case))}
    if case["op"] == "attn":
        H, N, D, P, per = case["heads"], case["kv_heads"], case["dim"], case["prefix"], _lengths(case)
        T = sum(q for q, _ in per)
        pairs = T * P + sum(q * k - q * (q - 1) // 2 for q, k in per)
        return {"bytes": 4 * N * D * (P + sum(k for _, k in per)) + T * H * (4 * D + 4), "flops": 4 * pairs * H * D}
    B, n, V = case["seqs"], case["drafts"], case["vocab"]
    rows = (n + 1) + (0 if case["points"] else n) + 1
    return {"bytes": 4 * B * V * rows, "flops": 4 * B * V * rows}


# ---- the definitions in 64 bits --------------------------------------------------------------------------

def _norm64(v, kind, w, b):
    mean = v.mean(-1, keepdim=True) if kind == "layer" else 0.0
    var = ((v - mean) ** 2).mean(-1, keepdim=True)
    return (v - mean) / torch.sqrt(var + EPS) * w.double() + (0.0 if b is None else b.double())


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        h, x, step = [], [], 1024
        for t in range(0, case["tokens"], step):
            v = s["y"][t:t + step].double()
            if case["post"]:
                v = _norm64(v, case["kind"], s["post_w"], s.get("post_b"))
            if case["gate"] != "none":
                v = v * (s["gate"][t:t + step] if case["gate"] == "token" else s["gate"]).double()
            h.append(s["h"][t:t + step].double() * 0.9 + v)
            x.append(_norm64(h[-1], case["kind"], s["pre_w"], s.get("pre_b")))
        return {"h": torch.cat(h), "x": torch.cat(x)}
    if case["op"] == "lora":
        ids, ranks = s["ids"].tolist(), s["ranks"].tolist()
        scales = s["scales"].tolist()
        groups = {a: torch.tensor([t for t, i in enumerate(ids) if i == a], device="cuda") for a in set(ids) if a >= 0}
        out = []
        for m in s["mods"]:
            y = m["y0"].double()
            for a, at in groups.items():
                low = m["x"][at].double() @ m["a"][a, :ranks[a]].double().t().contiguous()
                y[at] += scales[a] * (low @ m["b"][a, :, :ranks[a]].double().t().contiguous())
            out.append(y.reshape(-1))
        return torch.cat(out)
    if case["op"] == "attn":
        H, N, D, P = case["heads"], case["kv_heads"], case["dim"], case["prefix"]
        out, lse = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
        at = 0
        for b, (nq, nk) in enumerate(_lengths(case)):
            allowed = torch.ones((nq, P + nk), dtype=torch.bool, device="cuda").tril(P + nk - nq)
            for head in range(H):
                k = torch.cat([s["k_prefix"][:, head * N // H], s["k"][b, :nk, head * N // H]]).double()
                v = torch.cat([s["v_prefix"][:, head * N // H], s["v"][b, :nk, head * N // H]]).double()
                sc = (s["q"][at:at + nq, head].double() @ k.t().contiguous()) / math.sqrt(D)
                sc[~allowed] = -math.inf
                lse[at:at + nq, head] = torch.logsumexp(sc, -1)
                out[at:at + nq, head] = torch.softmax(sc, -1) @ v
            at += nq
        return {"out": out, "lse": lse}
    logp = torch.zeros((case["seqs"], case["drafts"] + 1), dtype=torch.float64)
    u, counts, temps, tokens = (s[k].tolist() for k in ("uniform", "counts", "temperature", "tokens"))
    for b in range(case["seqs"]):
        def dist(row):
            if temps[b] == 0:
                one = torch.zeros(case["vocab"], dtype=torch.float64, device="cuda")
                one[int(row.argmax())] = 1.0
                return one
            return torch.softmax(row.double() / temps[b], -1)
        for i in range(counts[b] + 1):
            p = dist(s["target"][b, i])
            if i == counts[b]:
                left = p
            else:
                x = tokens[b][i]
                if s["draft"] is None:
                    q = torch.zeros_like(p)
                    q[x] = 1.0
                else:
                    q = dist(s["draft"][b, i])
                if u[b][i] * float(q[x]) < float(p[x]):
                    logp[b, i] = math.log(float(p[x]))
                    continue
                left = torch.clamp(p - q, min=0.0)
                left = left if float(left.max()) > 0 else p
            x = int((left / s["noise"][b].double()).argmax())
            logp[b, i] = math.log(float(p[x]))
            break
    return {"out": None, "accepted": None, "logp": logp}
