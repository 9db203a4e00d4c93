"""What a serving step does with a paged cache and with its logits, as measurable cases: queries and keys with head
norms and positions, appended page by page; attention of the newest tokens over those pages; log probabilities of given
tokens with entropy and alternatives.  Through the entry points of paper_2608_12114_amd.wsr (`own`) or in plain torch
operations.

Sizes are those of the 8B- and 70B-shaped models this library sweeps (32 or 64 heads of 128 over 8 key heads, vocabulary
128256) and odd ones beside them.  Inputs come from torch's seeded generator; how long and how many things are follows
from the case alone."""
import math
import random

import torch

own = False
EPS = 1e-6


def listed():
    return [
        # one new token of one request, 8B heads, no head norms: latency alone
        {"name": "append_1seq_8b", "op": "append", "fmt": "f16", "seqs": 1, "queries": 1, "len": 300, "heads": 32,
         "kv_heads": 8, "dim": 128, "rot": 128, "pairs": False, "norm": "none", "axes": 1, "page": 16, "order": "token"},
        # a serving batch, 70B heads, queries and keys normed
        {"name": "append_64seq_70b", "op": "append", "fmt": "bf16", "seqs": 64, "queries": 1, "len": 500, "heads": 64,
         "kv_heads": 8, "dim": 128, "rot": 128, "pairs": False, "norm": "rms", "axes": 1, "page": 32, "order": "head"},
        # chunks of prompts with images: three position axes, layer norms with biases, half of a head turned, odd pages
        {"name": "append_3seq_601q_layer", "op": "append", "fmt": "f16", "seqs": 3, "queries": 601, "len": 1203, "heads": 12,
         "kv_heads": 4, "dim": 64, "rot": 32, "pairs": True, "norm": "layer", "axes": 3, "page": 7, "order": "token"},
        # prompts of a model of several modalities, 8B heads, normed
        {"name": "append_5seq_1800q_8b", "op": "append", "fmt": "bf16", "seqs": 5, "queries": 1800, "len": 1800, "heads": 32,
         "kv_heads": 8, "dim": 128, "rot": 128, "pairs": False, "norm": "rms", "axes": 3, "page": 16, "order": "token"},
        # one request early in its answer: the smallest call
        {"name": "paged_1seq_500", "op": "paged", "fmt": "f16", "seqs": 1, "queries": 1, "len": 500, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 16, "order": "token"},
        # a serving batch of requests of every length
        {"name": "paged_32seq_4096", "op": "paged", "fmt": "bf16", "seqs": 32, "queries": 1, "len": 4096, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 16, "order": "token"},
        # long documents, 70B heads
        {"name": "paged_7seq_65536", "op": "paged", "fmt": "bf16", "seqs": 7, "queries": 1, "len": 65536, "heads": 64,
         "kv_heads": 8, "dim": 128, "page": 64, "order": "head"},
        # four drafts and the last token of each request, pages of an odd size
        {"name": "paged_24seq_5q_6001", "op": "paged", "fmt": "f16", "seqs": 24, "queries": 5, "len": 6001, "heads": 64,
         "kv_heads": 8, "dim": 128, "page": 25, "order": "token"},
        # chunks of two prompts behind what is cached
        {"name": "paged_2seq_512q_4608", "op": "paged", "fmt": "bf16", "seqs": 2, "queries": 512, "len": 4608, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 32, "order": "token"},
        # one step's token with five alternatives
        {"name": "logp_1row_128256_5", "op": "logp", "rows": 1, "vocab": 128256, "top": 5, "heat": False},
        # a serving batch with twenty alternatives, sampled at its requests' temperatures
        {"name": "logp_64row_128256_20", "op": "logp", "rows": 64, "vocab": 128256, "top": 20, "heat": True},
        # a prompt scored, an odd vocabulary
        {"name": "logp_2055row_50257_1", "op": "logp", "rows": 2055, "vocab": 50257, "top": 1, "heat": False},
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _odd(rng, lo, hi):
    return min(int(_log(rng, lo, hi + 1)) | 1, hi)


HEADS = ((32, 8), (64, 8), (32, 32), (12, 4), (7, 1))


def draw(rng):
    op = rng.choice(("append", "paged", "logp"))
    if op == "logp":
        vocab = rng.choice((128256, 32000, _odd(rng, 1001, 151937)))
        return {"op": op, "rows": min(_odd(rng, 1, 4001), 2055 * 50257 // vocab), "vocab": vocab,
                "top": rng.choice((0, 1, rng.randint(2, 20), rng.randint(21, 64))), "heat": rng.random() < 0.5}
    heads, kv = rng.choice(HEADS)
    case = {"op": op, "fmt": rng.choice(("f16", "bf16")), "heads": heads, "kv_heads": kv, "dim": rng.choice((64, 128, 128)),
            "page": rng.choice((16, 16, 32, 64, rng.randint(1, 100))), "order": rng.choice(("token", "token", "head"))}
    if op == "append":
        queries = rng.choice((1, 1, _odd(rng, 2, 16), _odd(rng, 17, 1801)))
        seqs = _odd(rng, 1, 255) if queries < 17 else rng.randint(1, 2)
        rot = rng.choice((case["dim"], case["dim"], 8 * rng.randint(1, case["dim"] // 8)))
        return dict(case, seqs=seqs, queries=queries, len=queries + int(_log(rng, 1, 500)) - 1, rot=rot,
                    pairs=rng.random() < 0.3, norm=rng.choice(("none", "rms", "rms", "layer")), axes=rng.choice((1, 1, 3)))
    queries = rng.choice((1, 1, 1, _odd(rng, 2, 16), _odd(rng, 17, 512)))
    seqs = rng.choice((1, _odd(rng, 2, 64))) if queries < 17 else rng.randint(1, 2)
    room = 2 ** 28 // (seqs * kv * case["dim"])            # keys of the longest sequence, so that all fit the largest case
    most = min(room, 65536) if queries == 1 else min(room, 6001) if queries < 17 else 4608 - queries
    return dict(case, seqs=seqs, queries=queries, len=queries + _odd(rng, 1, most) - 1)


# ---- what follows from the case alone ----------------------------------------------------------------

def _half(case):
    return torch.bfloat16 if case["fmt"] == "bf16" else torch.float16


def _lengths(case):
    """[(queries, keys)] of each sequence, its queries the last of its keys; the first is as long as the case says."""
    r, out = random.Random(104729 * case["seqs"] + case["len"]), [(case["queries"], case["len"])]
    for _ in range(case["seqs"] - 1):
        n = case["queries"] if case["queries"] < 17 else r.randint(case["queries"] // 4, case["queries"])
        out.append((n, r.randint(n, max(n, case["len"]))))
    return out


def _row(case):
    """Entries of a row of the table: pages of the longest sequence and of the tokens to come."""
    return -(-(case["len"] + 64) // case["page"])


# ---- inputs, from the seed alone -----------------------------------------------------------------------

def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, to=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(to)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    if case["op"] == "logp":
        R, V = case["rows"], case["vocab"]
        logits = normal(R, V, std=2.5)
        # every eighth row is held to half of the vocabulary
        logits[5::8, V // 2:] = -math.inf
        heat = torch.tensor([(1.0, 0.7, 0.9, 1.3)[r % 4] for r in range(R)], dtype=torch.float32, device="cuda")
        scaled = logits / heat[:, None] if case["heat"] else logits
        noise = torch.empty_like(logits).exponential_(generator=g).clamp_(min=1e-30).log_()
        s = {"logits": logits, "tokens": (scaled - noise).argmax(-1).to(torch.int32)}
        return dict(s, heat=heat) if case["heat"] else s

    H, N, D, h, per = case["heads"], case["kv_heads"], case["dim"], _half(case), _lengths(case)
    starts = [sum(q for q, _ in per[:i]) for i in range(len(per) + 1)]
    # pages lie in the pool as requests came and went; entries that a sequence has not reached are -1
    used = [-(-k // case["page"]) for _, k in per]
    pool = sum(used) + max(4, sum(used) // 16)
    perm = torch.randperm(pool, device="cuda", generator=g)
    entry = torch.arange(_row(case), device="cuda")
    first = torch.tensor([sum(used[:i]) for i in range(len(used))], device="cuda")
    table = torch.where(entry < torch.tensor(used, device="cuda")[:, None], perm[(first[:, None] + entry).clamp(max=pool - 1)], -1)
    shape = (pool, N, case["page"], D) if case["order"] == "head" else (pool, case["page"], N, D)
    s = {"starts": ints(starts), "lens": ints([k for _, k in per]), "table": table.to(torch.int32),
         "k_cache": normal(*shape, to=h), "v_cache": normal(*shape, to=h)}
    T = starts[-1]
    if case["op"] == "paged":
        return dict(s, q=normal(T, H, D, std=2.5, to=h))
    s.update(q=normal(T, H * D), k=normal(T, N * D), v=normal(T, N * D))
    if case["norm"] != "none":
        s.update(q_w=normal(D, std=0.2, mean=1.0, to=h), k_w=normal(D, std=0.2, mean=1.0, to=h))
    if case["norm"] == "layer":
        s.update(q_b=normal(D, std=0.1, to=h), k_b=normal(D, std=0.1, to=h))
    half = case["rot"] // 2
    s["freqs"] = (500000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)).float()
    if case["axes"] > 1:
        # text counts on along all axes; a stretch of each chunk is an image, its rows and columns the other two
        place = torch.cat([torch.arange(k - q, k, device="cuda") for q, k in per])
        image = place % 7 > 2
        s["positions"] = torch.stack([torch.where(image, place - place % 7, place), torch.where(image, place // 24 % 24, place),
                                      torch.where(image, place % 24, place)]).to(torch.int32)
        s["axis_of"] = ints([(0, 0, 1, 2)[4 * i // half] for i in range(half)])
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:                      # the structures and the workspace that a program keeps beside its buffers
        from paper_2608_12114_amd import wsr
        _handles(wsr, s, case)
    return s


def _handles(wsr, s, case):
    new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if case["op"] == "logp":
        R, V, n = case["rows"], case["vocab"], case["top"]
        f32, i32 = torch.float32, torch.int32
        s["logp"], s["entropy"], s["rank"] = new(R, dtype=f32), new(R, dtype=f32), new(R, dtype=i32)
        s["top"], s["top_logp"] = new(R, n, dtype=i32), new(R, n, dtype=f32)
        s["handle"] = wsr.make_logprobs(
            n_rows=R, vocab=V, n_top=n, logits=s["logits"], row_stride=4 * V, tokens=s["tokens"], temperature=s.get("heat"),
            logp=s["logp"], rank=s["rank"], entropy=s["entropy"], top=s["top"], top_logp=s["top_logp"])
        s["ws"] = new(wsr.wsr_logprobs_workspace_bytes(s["handle"]), dtype=torch.uint8)
        return
    H, N, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    code = wsr.WSR_BF16 if case["fmt"] == "bf16" else wsr.WSR_F16
    head = case["order"] == "head"
    s["pages"] = wsr.make_pages(
        k=s["k_cache"], v=s["v_cache"], n_pages=s["k_cache"].shape[0], page_size=page, page_stride=2 * page * N * D,
        tok_stride=2 * D if head else 2 * N * D, head_stride=2 * page * D if head else 2 * D, table=s["table"],
        table_stride=4 * s["table"].shape[1], max_pages=s["table"].shape[1])
    T = s["q"].shape[0]
    s["out"] = new(T, H, D, dtype=_half(case))
    if case["op"] == "append":
        s["handle"] = wsr.make_qkv(
            fmt=code, kind=wsr.WSR_NORM_LAYER if case["norm"] == "layer" else wsr.WSR_NORM_RMS, eps=EPS,
            flags=(wsr.WSR_QKV_NORM if case["norm"] != "none" else 0) | (wsr.WSR_QKV_PAIRS if case["pairs"] else 0),
            n_heads=H, n_kv_heads=N, head_dim=D, rot_dim=case["rot"], n_axes=case["axes"], n_seqs=case["seqs"], n_tokens=T,
            q=s["q"], q_tok_stride=4 * H * D, k=s["k"], k_tok_stride=4 * N * D, v=s["v"], v_tok_stride=4 * N * D,
            q_w=s.get("q_w"), q_b=s.get("q_b"), k_w=s.get("k_w"), k_b=s.get("k_b"), freqs=s["freqs"], axis_of=s.get("axis_of"),
            positions=s.get("positions"), pos_axis_stride=4 * T, starts=s["starts"], lens=s["lens"], q_out=s["out"],
            q_out_tok_stride=2 * H * D, q_out_head_stride=2 * D, cache=s["pages"])
        return
    s["lse"] = new(T, H, dtype=torch.float32)
    s["handle"] = wsr.make_paged(
        fmt=code, n_heads=H, n_kv_heads=N, head_dim=D, n_seqs=case["seqs"], n_tokens=T, scale=D ** -0.5,
        max_len=page * s["table"].shape[1], q=s["q"], q_tok_stride=2 * H * D, q_head_stride=2 * D, starts=s["starts"],
        lens=s["lens"], out=s["out"], out_tok_stride=2 * H * D, out_head_stride=2 * D, lse=s["lse"], cache=s["pages"])
    s["ws"] = new(wsr.wsr_paged_workspace_bytes(s["handle"]), dtype=torch.uint8)


# ---- the measured calls --------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"append": _append, "paged": _paged, "logp": _logp}[op](s)
    from paper_2608_12114_amd import wsr
    stream = torch.cuda.current_stream()
    if op == "append":
        wsr.wsr_append_qkv(s["handle"], stream)
        return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if op == "paged":
        wsr.wsr_paged_attention(s["handle"], s["ws"], s["ws"].numel(), stream)
        return {"out": s["out"], "lse": s["lse"]}
    wsr.wsr_token_logprobs(s["handle"], s["ws"], s["ws"].numel(), stream)
    return {"logp": s["logp"], "rank": s["rank"], "entropy": s["entropy"], "top": s["top"], "top_logp": s["top_logp"]}


def _places(s, T):
    """Each token's sequence and place in it."""
    counts = (s["starts"][1:] - s["starts"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(s["case"]["seqs"], device="cuda"), counts, output_size=T)
    return seq, s["lens"][seq].long() - s["starts"][seq + 1].long() + torch.arange(T, device="cuda")


def _append(s):
    c = s["case"]
    H, N, D, half, T = c["heads"], c["kv_heads"], c["dim"], c["rot"] // 2, s["q"].shape[0]
    seq, place = _places(s, T)
    at = s["positions"][s["axis_of"].long()] if c["axes"] > 1 else place.expand(half, T)
    angle = at.t().double() * s["freqs"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turned(x, w, b):
        if c["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        x = x if b is None else x + b.float()
        x, rest = x[..., :2 * half], x[..., 2 * half:]
        u, v = (x[..., ::2], x[..., 1::2]) if c["pairs"] else (x[..., :half], x[..., half:])
        u, v = u * cos - v * sin, v * cos + u * sin
        x = torch.stack([u, v], -1).flatten(-2) if c["pairs"] else torch.cat([u, v], -1)
        return torch.cat([x, rest], -1).to(_half(c))

    page, slot = s["table"][seq, place // c["page"]].long(), place % c["page"]
    kc, vc = ((t.transpose(1, 2) if c["order"] == "head" else t) for t in (s["k_cache"], s["v_cache"]))
    kc[page, slot] = turned(s["k"].view(T, N, D), s.get("k_w"), s.get("k_b"))
    vc[page, slot] = s["v"].view(T, N, D).to(_half(c))
    return {"q": turned(s["q"].view(T, H, D), s.get("q_w"), s.get("q_b")), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _paged(s):
    c = s["case"]
    T, H, D = s["q"].shape
    N, B, n, G = c["kv_heads"], c["seqs"], c["queries"], c["heads"] // c["kv_heads"]
    seq, place = _places(s, T)
    i = torch.arange(n, device="cuda")
    first, counts = s["starts"][:-1].long(), (s["starts"][1:] - s["starts"][:-1]).long()

    def gathered(t):             # (B, N, keys, D), every sequence as long as the table's row
        t = t.transpose(1, 2) if c["order"] == "head" else t
        return t[s["table"].clamp(min=0).long()].flatten(1, 2).transpose(1, 2).float().contiguous()

    # queries padded to the longest chunk
    q = s["q"][(first[:, None] + i).clamp(max=T - 1)].float().view(B, n, N, G, D).transpose(1, 2).reshape(B, N, n * G, D)
    k = gathered(s["k_cache"])
    a = (q @ k.transpose(2, 3).contiguous()).view(B, N, n, G, -1) * D ** -0.5
    seen = torch.arange(k.shape[2], device="cuda") < ((s["lens"].long() - counts)[:, None] + i + 1).clamp(min=1)[..., None]
    a = a.masked_fill(~seen[:, None, :, None], -math.inf)
    m = a.amax(-1, keepdim=True)
    a = torch.exp(a - m)
    total = a.sum(-1, keepdim=True)
    v = gathered(s["v_cache"]).masked_fill(~seen[:, -1:, :, None], 0.0)
    o = (a.view(B, N, n * G, -1) @ v).view(B, N, n, G, D) / total
    j = torch.arange(T, device="cuda") - first[seq]
    out, lse = o[seq, :, j], (m + torch.log(total))[seq, :, j]
    return {"out": out.reshape(T, H, D).to(s["q"].dtype), "lse": lse.reshape(T, H)}


def _logp(s):
    c, logits = s["case"], s["logits"]
    pick = s["tokens"].long()[:, None]
    v = logits / s["heat"][:, None] if c["heat"] else logits
    v = v - v.amax(-1, keepdim=True)
    e = torch.exp(v)
    total = e.sum(-1, keepdim=True)
    logp = v - torch.log(total)
    mine = logits.gather(-1, pick)
    before = (logits == mine) & (torch.arange(c["vocab"], device="cuda") < pick)
    entropy = torch.log(total)[:, 0] - (e * v.masked_fill(e == 0, 0.0)).sum(-1) / total[:, 0]
    top = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
    return {"logp": logp.gather(-1, pick)[:, 0], "rank": ((logits > mine) | before).sum(-1).int(), "entropy": entropy,
            "top": top.int(), "top_logp": logp.gather(-1, top)}


# ---- what a pass cannot do without ---------------------------------------------------------------------

def work(case):
    if case["op"] == "logp":
        R, V = case["rows"], case["vocab"]
        return {"bytes": 4 * R * V + 8 * R * (2 + case["top"]), "flops": 6 * R * V}
    H, N, D, per = case["heads"], case["kv_heads"], case["dim"], _lengths(case)
    T = sum(q for q, _ in per)
    if case["op"] == "append":
        return {"bytes": 6 * T * D * (H + 2 * N) + 4 * T * case["axes"], "flops": 10 * T * D * (H + N)}
    pairs = sum(q * k - q * (q - 1) // 2 for q, k in per)
    return {"bytes": 4 * N * D * sum(k for _, k in per) + T * H * (4 * D + 4), "flops": 4 * pairs * H * D}


# ---- the definitions in 64 bits --------------------------------------------------------------------------

def _append64(case, s):
    D, rot = case["dim"], case["rot"]
    order = [j for i in range(rot // 2) for j in ((2 * i, 2 * i + 1) if case["pairs"] else (i, i + rot // 2))]
    order = torch.tensor(order + list(range(rot, D)), device="cuda")      # pairs side by side, then what stays
    back = torch.argsort(order)
    caches = [(t.transpose(1, 2) if case["order"] == "head" else t).double() for t in (s["k_cache"], s["v_cache"])]
    table, queries, at = s["table"].tolist(), [], 0
    for b, (nq, nk) in enumerate(_lengths(case)):
        places = torch.arange(nk - nq, nk, device="cuda")
        axes = s["positions"][:, at:at + nq] if case["axes"] > 1 else places[None]
        which = s["axis_of"].tolist() if case["axes"] > 1 else [0] * (rot // 2)
        angle = torch.stack([axes[a].double() for a in which], -1) * s["freqs"].double()
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]

        def heads(x, w, bias):
            x = x[at:at + nq].double().view(nq, -1, D)
            if case["norm"] != "none":
                mean = x.mean(-1, keepdim=True) if case["norm"] == "layer" else torch.zeros_like(x[..., :1])
                x = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + EPS) * s[w].double()
                x = x + s[bias].double() if bias in s else x
            x = x[..., order]
            z = torch.view_as_complex(x[..., :rot].reshape(nq, -1, rot // 2, 2).contiguous()) * turn
            return torch.cat([torch.view_as_real(z).flatten(-2), x[..., rot:]], -1)[..., back]

        queries.append(heads(s["q"], "q_w", "q_b"))
        pages = torch.tensor([table[b][p // case["page"]] for p in range(nk - nq, nk)], device="cuda")
        caches[0][pages, places % case["page"]] = heads(s["k"], "k_w", "k_b")
        caches[1][pages, places % case["page"]] = s["v"][at:at + nq].double().view(nq, -1, D)
        at += nq
    k, v = ((t.transpose(1, 2) if case["order"] == "head" else t).contiguous() for t in caches)
    return {"q": torch.cat(queries), "k_cache": k, "v_cache": v}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "append":
        return _append64(case, s)
    if case["op"] == "logp":
        logp, entropy, top_logp = [], [], []
        for r in range(case["rows"]):
            v = s["logits"][r].double() / (float(s["heat"][r]) if case["heat"] else 1.0)
            v = v - torch.logsumexp(v, -1)
            p = torch.exp(v)
            logp.append(v[s["tokens"][r].long()])
            entropy.append(-torch.special.xlogy(p, p).sum())
            top_logp.append(torch.topk(v, case["top"]).values)
        return {"logp": torch.stack(logp), "rank": None, "entropy": torch.stack(entropy), "top": None, "top_logp": torch.stack(top_logp)}
    H, N, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse, at = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda"), 0
    for b, (nq, nk) in enumerate(_lengths(case)):
        allowed = torch.ones((nq, nk), dtype=torch.bool, device="cuda").tril(nk - nq)
        pages = s["table"][b, :-(-nk // case["page"])].long()
        for head in range(N):
            k, v = ((t[pages, head] if case["order"] == "head" else t[pages, :, head]).flatten(0, 1)[:nk].double()
                    for t in (s["k_cache"], s["v_cache"]))
            for h in range(head * H // N, (head + 1) * H // N):
                sc = (s["q"][at:at + nq, h].double() @ k.t().contiguous()) / math.sqrt(D)
                sc[~allowed] = -math.inf
                lse[at:at + nq, h] = torch.logsumexp(sc, -1)
                out[at:at + nq, h] = torch.softmax(sc, -1) @ v
        at += nq
    return {"out": out, "lse": lse}
